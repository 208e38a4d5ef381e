"""The losses on the GPU, against the 64-bit oracle. Tolerances count roundings: u = 2^-24 is half a step of fp32."""
import math
import threading

import numpy as np
import pytest
import torch

from oracle import loss_oracle as O
from tests.harness import have_gpu, rng

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs an MI355X GPU")]

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
HALF = {F32: U, BF16: 2.0 ** -8}        # half a step, relative


def _M():
    from paper_2609_15037_amd import moara as M
    return M


def _L():
    from paper_2609_15037_amd import losses as L
    return L


def _np(t):
    return t.detach().double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _gpu(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _close(got, want, tol, what=""):
    """Same NaN and infinities, the others within tol (an array)."""
    got, want, tol = np.asarray(got, float), np.asarray(want, float), np.broadcast_to(tol, np.shape(want))
    assert got.shape == want.shape, what
    assert (np.isnan(got) == np.isnan(want)).all(), what
    inf = np.isinf(want)
    assert (got[inf] == want[inf]).all() and np.isfinite(got[~inf & ~np.isnan(want)]).all(), what
    ok = np.isfinite(want)
    assert not np.isnan(tol[ok]).any(), what
    off = np.abs(got[ok] - want[ok])
    bad = off > tol[ok]
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst by {np.max(off[bad] / np.maximum(tol[ok][bad], 1e-300)):.2f} " \
        f"times the tolerance ({off[bad].max():.3e})"


# ---------------------------------------------------------------- log-probabilities of tokens
# With a = scale (x - max): the difference, the factor and their product are rounded (3 u |a| in the exponent), the
# exponential is good to a step (2 u), and a sum adds u for each of the terms that one lane adds up (a row is on at least 16
# lanes, on 64 above a vocabulary of 1024, on 256 above 4096, or from 2048 rows on above 10240) and two for each 16 of them where its maximum moves. So e_j is good to
# (3 |a_j| + 2) u, their sum to s = (3 sum p_j |a_j| + 2 + n) u; log1p to two steps (4 u).
# The label is apart from the others' sum R, whose own error over the whole sum S is that of its terms alone: with d e_j <=
# (3 |a_j| + 2 + n) u e_j, d R / S <= sum over j != label of p_j (3 |a_j| + 2 + n) u =: o. It is what log S = log1p(R + e - 1)
# is off by, besides the label's own p (3 |a| + 2) u (0 where the label is the largest: e is 1), and 1 - p = R / S is off by
# d R / S + (R / S) (d S / S) <= o + (1 - p) s. (A sum over all j times 1 - p, which stood here first, is less than o: where
# p is nearly 1, R may be one term with |a| = 19, good to 59 u, when sum p |a| is nearly 0.)
# All this holds for numbers that fp32 holds to 24 bits. An exponential under 2^-126 may be taken as 0 or have fewer: V of
# them are off by at most V 2^-126 in R, and so in log p, which is as small there.

def _adds(shape):
    V, rows = shape[-1], np.prod(shape[:-1])
    return V / (16 if V <= 1024 else 64 if V <= 4096 or (V <= 10240 and rows >= 2048) else 256) * 1.125 + 12


def _others(a, p, lab):
    """o of the text above, for each row."""
    each = np.where(np.arange(a.shape[-1]) == lab[..., None], 0, p) * (3 * np.where(p > 0, np.abs(a), 0) + 2 + _adds(a.shape))
    return each.sum(axis=-1) * U


def _terms(x, scale):
    """a, log p, p, and the sum's relative error."""
    V = x.shape[-1]
    with np.errstate(all="ignore"):
        a = scale * (x - x.max(axis=-1, keepdims=True))
        log = O.log_softmax(scale * x)
        p = np.exp(log)
    n = _adds(x.shape)
    s = (3 * np.abs(O.xlogy(p, a)).sum(axis=-1) + 2 + n) * U
    return a, log, p, s


def _logps_tol(x, lab, scale):
    a, log, p, s = _terms(x, scale)
    on = (lab >= 0) & (lab < x.shape[-1])
    at = np.where(on, lab, 0)[..., None]
    al, ll, pl = (np.take_along_axis(t, at, -1)[..., 0] for t in (a, log, p))
    with np.errstate(all="ignore"):
        lse = -log.max(axis=-1)         # less the largest logit
        own = 2 * np.abs(al) * U + _others(a, p, lab) + pl * (3 * np.abs(al) + 2) * U * (np.abs(al) > 0) + 4 * U * np.abs(lse) + U * np.abs(ll)
        w = p * (1 + np.abs(np.where(p > 0, log, 0))) * (np.where(p > 0, 3 * np.abs(a), 0) + 4)
    H = np.abs(O.xlogy(p, log).sum(axis=-1))
    bits = w.sum(axis=-1) * U + (1 + H + np.abs(lse)) * s + 8 * U * (H + np.abs(lse))
    least = x.shape[-1] * 2.0 ** -126
    return np.where(on, own, 0) + least, np.where(on, bits, 0) + 200 * least, s


def _grad_tol(x, lab, g, h, scale, want, dtype):
    """p_j c with p_j from a rounded exponent and the sum, c from g, h and the entropy; then rounded to the type. An
    exponential under 2^-126 is 0."""
    a, log, p, s = _terms(x, scale)
    _, bits, _ = _logps_tol(x, lab, scale)
    h = np.zeros_like(g) if h is None else h
    H = np.abs(O.xlogy(p, log).sum(axis=-1))
    with np.errstate(all="ignore"):
        al, ll = (np.where(p > 0, np.abs(t), 0) for t in (a, log))
    g, h, H, bits = (t[..., None] for t in (np.abs(g), np.abs(h), H, bits))
    size = scale * p * (g + h * (H + ll))
    lse = np.abs(log.max(axis=-1, keepdims=True))
    tol = size * ((2 * al + 2 * ll + 3 * lse + 10) * U + s[..., None]) + scale * p * h * bits
    hit = np.arange(x.shape[-1]) == lab[..., None]
    tol = np.where(hit, tol + scale * g * (_others(a, p, lab)[..., None] + (1 - p) * (s[..., None] + 6 * U)), tol)
    tol = np.where(((lab >= 0) & (lab < x.shape[-1]))[..., None], tol, 0)
    return tol + HALF[dtype] * np.abs(want) + 2.0 ** -126 * scale * (g + 200 * h) + 2.0 ** -133


def _case(seed, T, V, dtype, scale=1.0, spread=2.0, gap=0, shift=0):
    """Logits (rows `gap` elements further apart, beginning `shift` elements into a buffer), labels, gradients."""
    r = rng(7, seed, T, V)
    x = spread * r.standard_normal((T, V))
    lab = r.integers(0, V, T)
    lab[r.random(T) < 0.2] = -100
    if T > 2:
        lab[0], lab[1], lab[2] = 0, V - 1, V
    for t in range(T):      # labels of every probability, some nearly 1
        if 0 <= lab[t] < V:
            x[t, lab[t]] += r.choice([0.0, 4.0, 9.0, 20.0])
    ld = V + gap
    buf = torch.full((shift + T * ld + 8,), 77.0, dtype=dtype, device="cuda")
    view = buf[shift:shift + T * ld].view(T, ld)[:, :V]
    view.copy_(_gpu(x))
    g, h = (r.standard_normal(T) * r.choice([0.0, 1.0, 1e-3], T) for _ in range(2))
    return view, _gpu(lab), _gpu(g, F32), _gpu(h, F32)


def _check_logps(x, lab, g, h, scale=1.0, entropy=True, back=None):
    """Forward and backward against the oracle; back: the call that gives the gradient."""
    M = _M()
    s32 = float(np.float32(scale))
    X, labels, V = _np(x).reshape(-1, x.shape[-1]), _np(lab).reshape(-1), x.shape[-1]
    logp, H, stats = M.moara_token_logps(x, lab, scale=scale, entropy=entropy)
    want, wantH = O.token_logps(X, labels, s32)
    tol, tolH, _ = _logps_tol(X, labels, s32)
    _close(_np(logp).reshape(-1), want, tol, "logp")
    if entropy:
        _close(_np(H).reshape(-1), wantH, tolH, "entropy")
        again = M.moara_token_logps(x, lab, scale=scale)
        assert again[1] is None and torch.equal(again[0].nan_to_num(nan=7e7), logp.nan_to_num(nan=7e7))     # NaN is not itself
    kw = dict(entropy=H, grad_entropy=h) if entropy else {}
    grad = M.moara_token_logps_backward(x, lab, stats, g, scale=scale, **kw) if back is None else back(stats, kw)
    assert grad.dtype == x.dtype and grad.shape == x.shape
    gn, hn = _np(g).reshape(-1), _np(h).reshape(-1) if entropy else None
    ref = O.token_logps_grad(X, labels, gn, hn, s32)
    _close(_np(grad).reshape(-1, V), ref, _grad_tol(X, labels, gn, hn, s32, ref, x.dtype), "gradient")
    return logp, H, stats, grad


SIZES = [1, 2, 3, 4, 5, 7, 8, 9, 31, 63, 64, 65, 255, 256, 511, 512, 513, 2047, 2048, 2049, 4095, 8191, 8192, 8193]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", SIZES)
def test_logps_of_every_size(V, dtype):
    for seed, (T, scale, entropy, gap, shift) in enumerate([(7, 1.0, True, 0, 0), (5, 1.25, False, 3, 1), (1, 0.7, True, 0, 3),
                                                           (261, 1.0, False, 1, 0)]):
        if T * V > 1 << 21:
            T = 9
        x, lab, g, h = _case(seed, T, V, dtype, scale, gap=gap, shift=shift)
        _check_logps(x, lab, g, h, scale, entropy)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,V", [(3, 50021), (2, 131073), (33, 32000), (1, 131072), (600, 12289), (300, 70001)])
def test_logps_of_large_vocabularies(T, V, dtype):
    x, lab, g, h = _case(1, T, V, dtype, 1.0)
    _check_logps(x, lab, g, h)
    _check_logps(x, lab, g, h, entropy=False)


@pytest.mark.parametrize("T", [63, 64, 65, 255, 256, 257, 511, 513, 1025, 2049])
def test_logps_of_many_rows(T):
    """Row counts about those where the work is laid out otherwise; all rows are as those of a call on a few."""
    M = _M()
    for V in (300, 2500, 9000):
        x, lab, g, h = _case(T, T, V, BF16)
        logp, H, stats = M.moara_token_logps(x, lab, entropy=True)
        want, wantH = O.token_logps(_np(x), _np(lab))
        tol, tolH, _ = _logps_tol(_np(x), _np(lab), 1.0)
        _close(_np(logp), want, tol, "logp")
        _close(_np(H), wantH, tolH, "entropy")
        assert torch.equal(M.moara_token_logps(x, lab)[0], logp)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_logps_of_a_large_offset_and_a_large_spread(dtype):
    """Logits 10^4 from 0, logits whose exponentials underflow, and a label that has nearly all of the probability."""
    for V in (100, 5000):
        x, lab, g, h = _case(3, 12, V, dtype)
        _check_logps(x + 1e4, lab, g, h)
        _check_logps(x * 100, lab, g, h)
        _check_logps(x * 1e30, lab, g, h)
        y = torch.zeros(4, V, dtype=dtype, device="cuda")
        lab = torch.tensor([0, V // 2, V - 1, 1], device="cuda")
        y[torch.arange(4), lab] = torch.tensor([12.0, 30.0, 60.0, 100.0], device="cuda").to(dtype)
        logp = _check_logps(y, lab, g[:4].fill_(1.0), h[:4])[0]
        # relative accuracy where p is nearly 1
        want = -np.log1p((V - 1) * np.exp(-np.array([12.0, 30.0, 60.0])))
        np.testing.assert_allclose(_np(logp)[:3], want, rtol=1e-5)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [9, 700, 3000, 20000])
def test_logps_of_masked_and_bad_rows(V, dtype):
    """-inf and the type's lowest value in most places; rows with nothing left, NaN, +inf; bad values in rows without a label."""
    r = rng(5, V)
    x, lab, g, h = _case(4, 14, V, dtype)
    lab[:] = torch.from_numpy(r.integers(0, V, 14)).cuda()
    off = _gpu(r.random((14, V)) < 0.9)
    off[torch.arange(14), lab] = False
    x[0, off[0]] = -math.inf
    x[1, off[1]] = torch.finfo(dtype).min
    x[2] = -math.inf
    x[2, lab[2]] = 3.0                  # one word is left
    x[3, lab[3]] = -math.inf            # the label is not
    x[4] = -math.inf
    x[5, 1] = math.nan
    x[6, 2] = math.inf
    x[7] = torch.finfo(dtype).min       # all alike
    x[8] = math.nan
    x[9], x[10] = math.inf, -math.inf
    lab[8:11] = torch.tensor([-100, V, -1], device="cuda")
    x[11, off[11]] = torch.finfo(dtype).max
    g.fill_(0.5)
    h.fill_(0.25)
    logp, H, _, grad = _check_logps(x, lab, g, h)
    assert logp[2] == 0 and H[2] == 0 and not grad[2].any()
    assert logp[3] == -math.inf and torch.isfinite(grad[3]).all()
    assert logp[4:7].isnan().all() and H[4:7].isnan().all() and grad[4:7].isnan().all()
    assert not logp[8:11].any() and not H[8:11].any() and not grad[8:11].any()
    _check_logps(x, lab, g, h, entropy=False)
    g[4:7] = 0
    h[4:7] = 0
    M = _M()
    logp, H, stats = M.moara_token_logps(x, lab, entropy=True)
    assert not M.moara_token_logps_backward(x, lab, stats, g, entropy=H, grad_entropy=h)[4:7].any()    # no gradient, whatever the row


def test_logps_of_no_tokens_and_of_no_labels():
    M = _M()
    for dtype in (F32, BF16):
        x = torch.empty(0, 50, device="cuda", dtype=dtype)
        lab = torch.empty(0, dtype=torch.int64, device="cuda")
        logp, H, stats = M.moara_token_logps(x, lab, entropy=True)
        assert logp.numel() == 0 and M.moara_token_logps_backward(x, lab, stats, logp).shape == (0, 50)
        x = torch.full((5, 50), math.nan, device="cuda", dtype=dtype)
        lab = torch.full((5,), -100, device="cuda")
        logp, H, stats = M.moara_token_logps(x, lab, entropy=True)
        grad = M.moara_token_logps_backward(x, lab, stats, torch.ones(5, device="cuda"), entropy=H, grad_entropy=logp)
        assert not logp.any() and not H.any() and not grad.any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_logps_of_views_and_of_outputs_given(dtype):
    """Batches without their last position, every other row, transposed batches; the gradient in a given tensor between
    guards, and in place of the logits (padded rows too)."""
    M = _M()
    base = _case(6, 30, 2100, dtype, gap=11)[0]
    lab = torch.randint(-1, 2100, (30,), device="cuda")
    g, h = torch.randn(30, device="cuda"), torch.randn(30, device="cuda")
    _check_logps(base[::2], lab[::2].contiguous(), g[::2].contiguous(), h[::2].contiguous())
    b = torch.randn(5, 6, 2100, device="cuda").to(dtype)
    for v in (b[:, :-1], b[:, 1:], b[1:4, 2:3], b[::2, ::2], b.transpose(0, 1), b[:, :, 1:-3], b[2:3]):
        n = v.shape[0] * v.shape[1]
        lb = torch.randint(-1, v.shape[2], v.shape[:2], device="cuda")
        _check_logps(v, lb, g[:n].view(lb.shape).contiguous(), h[:n].view(lb.shape).contiguous())

    for off in (0, 1, 5):
        buf = torch.full((30 * 2100 + 16,), 55.0, dtype=dtype, device="cuda")
        out = buf[off:off + 30 * 2100].view(30, 2100)
        _check_logps(base, lab, g, h, back=lambda stats, kw: M.moara_token_logps_backward(base, lab, stats, g, out=out, **kw))
        assert (buf[:off] == 55).all() and (buf[off + 30 * 2100:] == 55).all()

    def in_place(stats, kw):
        own = base.as_strided(base.shape, base.stride()).clone(memory_format=torch.preserve_format)
        wide = torch.full((30, 2111), 44.0, dtype=dtype, device="cuda")
        wide[:, :2100] = base
        view = wide[:, :2100]
        res = M.moara_token_logps_backward(view, lab, stats, g, out=view, **kw)
        assert res is view and (wide[:, 2100:] == 44).all()
        assert torch.equal(view, M.moara_token_logps_backward(own, lab, stats, g, **kw))
        return res
    _check_logps(base, lab, g, h, back=in_place)
    for bad in (base.float().double(), base[:, :-1], base[:29], torch.empty(30, 2200, dtype=dtype, device="cuda")[:, :2100],
                base.as_strided((30, 2100), (2100, 1))):
        with pytest.raises(ValueError):
            M.moara_token_logps_backward(base, lab, torch.empty(30, 4, device="cuda"), g, out=bad)


def test_logps_binding_refusals():
    M = _M()
    x, lab = torch.zeros(4, 9, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    stats, g = torch.zeros(4, 4, device="cuda"), torch.zeros(4, device="cuda")
    for a, b in ((x.half(), lab), (x.t(), lab), (x, lab.int()), (x, lab[:3]), (x, lab.cpu()), (x.cpu(), lab),
                 (x, torch.zeros(8, dtype=torch.int64, device="cuda")[::2])):
        with pytest.raises(ValueError):
            M.moara_token_logps(a, b)
    for s, gg, kw in ((stats[:3], g, {}), (stats, g.half(), {}), (stats, g[:2], {}), (stats, g, dict(grad_entropy=g)),
                      (stats, g, dict(grad_entropy=g[:2], entropy=g)), (stats, g, dict(grad_entropy=g, entropy=g.cpu()))):
        with pytest.raises(ValueError):
            M.moara_token_logps_backward(x, lab, s, gg, **kw)
    for scale in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(M.MoaraError):
            M.moara_token_logps(x, lab, scale=scale)
    with pytest.raises(M.MoaraError):
        M.moara_token_logps(x[:1].expand(4, 9), lab)


def test_logps_past_32_bits():
    """More elements than 32 bits count: the last rows as those of a call of their own, the first ones too."""
    M = _M()
    T, V = 33000, 131072
    x = torch.zeros(T, V, dtype=BF16, device="cuda")
    small = torch.randn(6, V, device="cuda").to(BF16)
    rows = torch.tensor([0, 1, 16383, 16384, 32768, T - 1], device="cuda")
    x[rows] = small
    lab = torch.full((T,), -100, device="cuda")
    lab[rows] = torch.tensor([0, 5, V - 1, 77, 99999, V - 2], device="cuda")
    g = torch.zeros(T, device="cuda")
    g[rows] = torch.arange(1.0, 7.0, device="cuda")
    logp, H, stats = M.moara_token_logps(x, lab, entropy=True)
    grad = M.moara_token_logps_backward(x, lab, stats, g)
    X, labels, gn = _np(small), _np(lab[rows]), _np(g[rows])
    (want, wantH), (tol, tolH, _) = O.token_logps(X, labels), _logps_tol(X, labels, 1.0)
    _close(_np(logp[rows]), want, tol, "logp")
    _close(_np(H[rows]), wantH, tolH, "entropy")
    ref = O.token_logps_grad(X, labels, gn)
    _close(_np(grad[rows]), ref, _grad_tol(X, labels, gn, None, 1.0, ref, BF16), "gradient")
    lab_off = torch.ones(T, dtype=torch.bool, device="cuda")
    lab_off[rows] = False
    assert not logp[lab_off].any()
    for a in range(0, T, 4096):
        keep = lab_off[a:a + 4096]
        assert not grad[a:a + 4096][keep].any()


# ---------------------------------------------------------------- packed sequences

def _offsets(r, S, T, kind):
    """Bounds of S sequences in T tokens."""
    if kind == "one each":
        return np.arange(S + 1)
    lo, hi = (0, T) if kind == "whole" else (T // 10, T - T // 7)
    if kind == "one long":          # all but the middle one have at most a token
        cuts = np.minimum(np.arange(S + 1), S // 2)
        return np.where(np.arange(S + 1) <= S // 2, cuts, T - (S - np.arange(S + 1)) // 2).clip(0, T)
    return np.concatenate([[lo], np.sort(r.integers(lo, hi + 1, S - 1)), [hi]])


LAYOUTS = [  # tokens, sequences, kind (None: equal lengths)
    (2, 2, None), (2, 2, "one each"), (1, 2, "whole"), (10, 4, "part"), (64, 2, None), (63 * 8, 8, None), (65 * 4, 4, None), (1000, 6, "whole"),
    (1023, 2, "whole"), (1024, 2, "whole"), (1025, 2, "part"), (2048, 2, None), (4096, 4, None), (5000, 130, "part"),
    (3000, 1000, "whole"), (3001, 3000, "whole"), (20000, 66, "one long"), (70001, 2, "part"), (300000, 4098, "whole"),
    (100000, 20, "one long"), (6, 600, "whole"), (0, 4, None), (0, 6, "whole")]


def _layout(seed, T, S, kind, mask):
    r = rng(11, seed, T, S)
    offsets = None if kind is None else _offsets(r, S, T, kind)
    on = None
    if mask != "none":
        on = r.random(T) < 0.6
        if mask == "empty rows":        # whole sequences, pairs among them, without a token
            o = np.arange(S + 1) * (T // S) if offsets is None else offsets
            for s in range(0, S, 3):
                on[o[s]:o[min(s + 2, S)]] = False
    shape = (S, T // S) if offsets is None else (T,)
    seqs = O.members(T, S, offsets, on)
    put = lambda a, dt=F32: _gpu(a.reshape(shape), dt)  # noqa: E731
    kw = dict(offsets=None if offsets is None else _gpu(offsets.astype(np.int64)), mask=None if on is None else put(on, None))
    return r, seqs, put, on, kw


def _spoil(r, x, seqs):
    """Values that nothing may depend on where no sequence has a token."""
    off = np.ones(x.size, bool)
    for t in seqs:
        off[t] = False
    x = x.astype(np.float32)
    x[off] = r.choice(np.float32([np.nan, np.inf, -np.inf, 3e38]), off.sum())
    return x


def _flat(t):
    return _np(t).reshape(-1)


PREFERENCES = [dict(), dict(smoothing=0.1, margin=0.5, beta=0.5), dict(average=True, beta=2.0, margin=0.2), dict(kind="hinge", beta=0.05),
               dict(kind="square", beta=0.3, average=True), dict(kind="hinge", average=True, margin=-0.4, beta=0.7)]


@pytest.mark.parametrize("T,S,kind", LAYOUTS)
@pytest.mark.parametrize("mask", ["none", "random", "empty rows"])
def test_preference_over_layouts(T, S, kind, mask):
    """Sums are 64 bits: what is left are the roundings to fp32 of a result (u) and of a slope before the mean (2 u), its
    product with the gradient (u); 64-bit sums over T tokens and the exponentials add less than 2^-40 of the terms."""
    M = _M()
    for i, spec in enumerate(PREFERENCES):
        r, seqs, put, on, kw = _layout(i, T, S, kind, mask)
        logp, ref = _spoil(r, -r.exponential(size=T), seqs), None if i == 1 else _spoil(r, -r.exponential(size=T), seqs)
        kinds = {"sigmoid": M.MOARA_PREF_SIGMOID, "hinge": M.MOARA_PREF_HINGE, "square": M.MOARA_PREF_SQUARE}
        cfg = M.moara_preference_default_config(**{**spec, "kind": kinds[spec.get("kind", "sigmoid")],
                                                   "average": int(spec.get("average", False))})
        gl = torch.tensor(0.37, device="cuda")
        out, rewards, slope = M.moara_preference_loss(cfg, put(logp), None if ref is None else put(ref), **kw)
        grad = M.moara_preference_loss_backward(cfg, put(logp), slope, gl, **kw)
        clean = lambda x: None if x is None else np.where(np.isfinite(x) & (np.abs(x) < 1e38), x, 0).astype(float)  # noqa: E731
        w_out, w_rewards, w_grad = O.preference(clean(logp), clean(ref), seqs, **spec)
        size = sum(np.abs(clean(logp)[t]).sum() for t in seqs) + 1
        _close(_np(out), w_out, 2 * U * np.abs(w_out) + 2.0 ** -40 * (np.abs(w_out) + spec.get("beta", 0.1) * size), f"out {spec}")
        _close(_np(rewards), w_rewards, 2 * U * np.abs(w_rewards) + 2.0 ** -40 * spec.get("beta", 0.1) * size, f"rewards {spec}")
        w_grad = w_grad * float(gl)
        _close(_flat(grad), w_grad, 5 * U * np.abs(w_grad) + 2.0 ** -40 * size * 4 + 2.0 ** -149 if spec.get("kind") == "square"
               else 5 * U * np.abs(w_grad) + 2.0 ** -149 + 2.0 ** -40 * np.abs(w_grad) * size, f"gradient {spec}")
        again = M.moara_preference_loss(cfg, put(logp), None if ref is None else put(ref), **kw)
        assert all(torch.equal(a, b) for a, b in zip(again, (out, rewards, slope)))


POLICIES = [dict(), dict(kl="exp", kl_coef=0.3, entropy_coef=0.02), dict(kl="linear", kl_coef=0.1, reduce="sequences"),
            dict(kl="square", kl_coef=0.2, reduce="sequences", divisor=12.0, entropy_coef=-0.1), dict(divisor=1e4, low=0.1, high=0.28),
            dict(low=1.0, high=math.inf, kl_coef=0.5)]


def _policy_cfg(M, spec, **kw):
    kls = {"exp": M.MOARA_KL_EXP, "linear": M.MOARA_KL_LINEAR, "square": M.MOARA_KL_SQUARE}
    return M.moara_policy_default_config(
        clip_low=spec.get("low", 0.2), clip_high=spec.get("high", 0.2), kl=kls[spec.get("kl", "exp")], kl_coef=spec.get("kl_coef", 0.0),
        entropy_coef=spec.get("entropy_coef", 0.0), divisor=spec.get("divisor", 0.0),
        reduce=M.MOARA_MEAN_SEQUENCES if spec.get("reduce") == "sequences" else M.MOARA_MEAN_TOKENS, **kw)


def _policy_tol(logp, old, ref, adv, entropy, seqs, spec):
    """d and q are exact differences rounded once (u of them in the exponent); expf and expm1f to two steps (4 u); a product
    with the advantage (u). e^q - q - 1 has its terms' errors where they are added (|q| >= 1/2: (5 u + u |q|) e^q + 2 u
    (|q| + 1)), a series of nine rounded steps below it. Weights 3 u, further products 4 u."""
    d = np.zeros_like(logp) if old is None else logp - old
    ratio = (np.abs(d) + 6) * U
    gain, slope, far, dfar, _, moved = O.policy_terms(logp, old, ref, adv, spec.get("low", 0.2), spec.get("high", 0.2), spec.get("kl", "exp"))

    def excess(q, f):
        return np.where(np.abs(q) < 0.51, 24 * U * f, 0) + np.where(np.abs(q) >= 0.49, (5 + np.abs(q)) * U * np.exp(q) + 3 * U * (np.abs(q) + 1), 0)
    q = np.zeros_like(logp) if ref is None else ref - logp
    kl = spec.get("kl", "exp")
    t_far = excess(q, np.abs(far)) if kl == "exp" else 4 * U * np.abs(far)
    t_dfar = (6 * U + U * np.abs(q)) * np.abs(dfar) + U * np.abs(q) * np.exp(q) if kl == "exp" else 3 * U * np.abs(dfar)
    w = O.policy_weights(seqs, spec.get("reduce", "tokens"), spec.get("divisor", 0.0))
    each = np.zeros_like(logp)
    for t, x in zip(seqs, w):
        each[t] = x
    mean = lambda x: float((each * x).sum())  # noqa: E731
    k, b = abs(spec.get("kl_coef", 0)), abs(spec.get("entropy_coef", 0))
    e = np.zeros_like(logp) if entropy is None else np.abs(entropy)
    t_out = np.array([0, mean(np.abs(gain) * ratio), mean(t_far), U * mean(e), U, mean(excess(d, moved))])
    t_out[0] = t_out[1] + k * t_out[2] + b * t_out[3] + 2 * U * (mean(np.abs(gain)) + k * mean(np.abs(far)) + b * mean(e))
    size = np.array([mean(np.abs(gain)) + k * mean(np.abs(far)) + b * mean(e), mean(np.abs(gain)), mean(np.abs(far)), mean(e), 1, mean(moved)])
    t_grad = each * (np.abs(slope) * (ratio + 8 * U) + k * (t_dfar + 8 * U * np.abs(dfar)))
    return t_out + size * (U + 2.0 ** -40), t_grad + 2.0 ** -149, 8 * U * each * b + 2.0 ** -149


@pytest.mark.parametrize("T,S,kind", LAYOUTS)
@pytest.mark.parametrize("mask", ["none", "random", "empty rows"])
def test_policy_over_layouts(T, S, kind, mask):
    M = _M()
    for i, spec in enumerate(POLICIES):
        r, seqs, put, on, kw = _layout(100 + i, T, S, kind, mask)
        base = -r.exponential(size=T)
        logp = _spoil(r, base, seqs)
        old = _spoil(r, base + 0.25 * r.standard_normal(T), seqs) if i % 3 else None
        ref = _spoil(r, base + r.choice([0.05, 1.0], T) * r.standard_normal(T), seqs) if spec.get("kl_coef") or i == 4 else None
        entropy = _spoil(r, r.exponential(size=T), seqs) if "entropy_coef" in spec else None
        whole = i % 2 == 0
        adv = r.standard_normal(S).astype(np.float32) * (r.random(S) < 0.9) if whole else _spoil(r, r.standard_normal(T), seqs)
        cfg = _policy_cfg(M, spec, sequence_advantages=int(whole))
        gl = torch.tensor([-1.7], device="cuda")
        opt = lambda x: None if x is None else put(x)  # noqa: E731
        args = dict(old_logp=opt(old), ref_logp=opt(ref), entropy=opt(entropy), **kw)
        a = _gpu(adv, F32) if whole else put(adv)
        out, weight = M.moara_policy_loss(cfg, put(logp), a, **args)
        grad, grad_entropy = M.moara_policy_loss_backward(cfg, put(logp), a, weight, gl, **args)
        clean = lambda x: None if x is None else np.where(np.isfinite(x) & (np.abs(x) < 1e38), x, 0).astype(float)  # noqa: E731
        per = np.zeros(T)
        if whole:
            for t, x in zip(seqs, adv):
                per[t] = x
        else:
            per = clean(adv)
        c = [clean(x) for x in (logp, old, ref)]
        spec_o = {k: v for k, v in spec.items()}
        w_out, w_weight, w_grad, w_ge = O.policy(*c, per, clean(entropy), seqs, **spec_o)
        t_out, t_grad, t_ge = _policy_tol(*c, per, clean(entropy), seqs, spec_o)
        _close(_np(out), w_out, t_out, f"out {spec}")
        _close(_np(weight)[:-1] * _np(weight)[-1], w_weight, 3 * U * w_weight, f"weight {spec}")
        _close(_flat(grad), -1.7 * w_grad, 1.7 * t_grad + 2 * U * np.abs(1.7 * w_grad), f"gradient {spec}")
        assert (grad_entropy is None) == (entropy is None)
        if entropy is not None:
            _close(_flat(grad_entropy), -1.7 * w_ge, 1.7 * t_ge, f"entropies' gradient {spec}")
        again = M.moara_policy_loss(cfg, put(logp), a, **args)
        assert torch.equal(again[0], out) and torch.equal(again[1], weight)


def test_policy_next_to_the_bounds():
    """Ratios a hair on either side of the bounds: log-probabilities that are neighbouring fp32 numbers decide."""
    M = _M()
    for low, high in ((0.2, 0.2), (0.1, 0.28), (0.5, 3.0)):
        d = []
        for bound in (math.log1p(high), math.log1p(-low)):
            x = np.float32(bound)
            for _ in range(3):
                x = np.nextafter(x, np.float32(-9))
            for _ in range(7):
                d.append(x)
                x = np.nextafter(x, np.float32(9))
        logp = np.array(d * 2, np.float32)
        adv = np.repeat(np.float32([1.0, -1.0]), len(d))
        cfg = M.moara_policy_default_config(clip_low=low, clip_high=high)
        out, weight = M.moara_policy_loss(cfg, _gpu(logp[None]), _gpu(adv[None]), old_logp=_gpu(np.zeros_like(logp)[None]))
        grad, _ = M.moara_policy_loss_backward(cfg, _gpu(logp[None]), _gpu(adv[None]), weight, torch.ones(1, device="cuda"),
                                               old_logp=_gpu(np.zeros_like(logp)[None]))
        clipped = ((logp.astype(float) > math.log1p(high)) & (adv > 0)) | ((logp.astype(float) < math.log1p(-low)) & (adv < 0))
        assert (_flat(grad) == 0).tolist() == clipped.tolist() and 0 < clipped.sum() < len(logp)
        assert float(out[4]) == pytest.approx(clipped.mean(), rel=2 * U)


def test_policy_of_extreme_ratios():
    """Overflowing ratios: bounded where the advantage is positive, the formula's infinity where it is not."""
    M = _M()
    logp, old = torch.tensor([[0.0, 0.0, -200.0, -200.0]], device="cuda"), torch.tensor([[-200.0, -200.0, 0.0, 0.0]], device="cuda")
    for adv, want in (([1.0, 0.0, 1.0, -1.0], None), ([1.0, -1.0, 1.0, -1.0], math.inf)):
        a = torch.tensor([adv], device="cuda")
        mask = torch.tensor([[True, adv[1] != 0, True, True]], device="cuda")
        cfg = M.moara_policy_default_config()
        out, w = M.moara_policy_loss(cfg, logp, a, old_logp=old, mask=mask)
        grad, _ = M.moara_policy_loss_backward(cfg, logp, a, w, torch.ones(1, device="cuda"), old_logp=old, mask=mask)
        if want is None:
            assert float(out[0]) == pytest.approx(-(1.2 + 0 - 0.8) / 3, rel=1e-6) and not grad.any()
        else:
            assert float(out[0]) == want and float(grad[0, 1]) == math.inf


@pytest.mark.parametrize("seed", range(4))
def test_falling_offsets_touch_nothing_else(seed):
    """Offsets that fall or leave the tokens: sums of whatever, but nothing outside the tensors is read or written."""
    M = _M()
    r = rng(17, seed)
    T, S = 3000, 64
    offsets = r.integers(-5, T + 5, S + 1) if seed % 2 else r.integers(-2 ** 60, 2 ** 60, S + 1)
    buf = torch.full((T + 200,), 9.0, device="cuda")
    logp = buf[100:100 + T]
    logp.copy_(_gpu(-r.exponential(size=T)))
    o = _gpu(offsets)
    cfg = M.moara_preference_default_config()
    out, rewards, slope = M.moara_preference_loss(cfg, logp, offsets=o)
    grad = M.moara_preference_loss_backward(cfg, logp, slope, torch.ones(1, device="cuda"), offsets=o)
    pol = M.moara_policy_default_config()
    _, w = M.moara_policy_loss(pol, logp, logp, offsets=o)
    M.moara_policy_loss_backward(pol, logp, logp, w, torch.ones(1, device="cuda"), offsets=o)
    bal = M.moara_balance_default_config(experts=8, top_k=1)
    x, i = torch.randn(T, 8, device="cuda"), torch.zeros(T, 1, dtype=torch.int32, device="cuda")
    _, _, sl = M.moara_balance_loss(bal, x, i, offsets=o)
    M.moara_balance_loss_backward(bal, x, sl, torch.ones(1, device="cuda"), offsets=o)
    torch.cuda.synchronize()
    assert grad.shape == (T,) and (buf[:100] == 9).all() and (buf[100 + T:] == 9).all()


def test_sequence_binding_refusals():
    M = _M()
    x, o = torch.zeros(12, device="cuda"), torch.tensor([0, 3, 6, 9, 12], device="cuda")
    cfg, pol = M.moara_preference_default_config(), M.moara_policy_default_config()
    rows = x.view(4, 3)
    for a, kw in ((x, {}), (rows, dict(offsets=o)), (x, dict(offsets=o.int())), (x, dict(offsets=o[::2])), (x.double(), dict(offsets=o)),
                  (x, dict(offsets=o.cpu())), (rows, dict(mask=torch.ones(12, dtype=torch.bool, device="cuda"))),
                  (rows, dict(mask=torch.ones(4, 3, device="cuda"))), (rows.t(), {})):
        with pytest.raises(ValueError):
            M.moara_preference_loss(cfg, a, **kw)
        with pytest.raises(ValueError):
            M.moara_policy_loss(pol, a, a, **kw)
    for kw in (dict(ref_logp=x), dict(ref_logp=rows.half()), dict(ref_logp=rows.cpu())):
        with pytest.raises(ValueError):
            M.moara_preference_loss(cfg, rows, **kw)
    for a, kw in ((x, {}), (rows[0], {}), (rows, dict(old_logp=x)), (rows, dict(entropy=rows.double()))):
        with pytest.raises(ValueError):
            M.moara_policy_loss(pol, rows, a, **kw)
    per = M.moara_policy_default_config(sequence_advantages=1)
    with pytest.raises(ValueError):
        M.moara_policy_loss(per, rows, rows)
    for bad in (o[:4], o[:1], o[:0]):           # three sequences, none, no offsets
        with pytest.raises(M.MoaraError):
            M.moara_preference_loss(cfg, x, offsets=bad)
    with pytest.raises(M.MoaraError):
        M.moara_policy_loss(M.moara_policy_default_config(kl_coef=0.1), rows, rows)


# ---------------------------------------------------------------- load balancing

def _balance_case(seed, T, E, k, S, kind, mask, dtype):
    r, seqs, _, on, kw = _layout(seed, T, S, kind, mask)
    x = _gpu(1.5 * r.standard_normal((T, E)) + r.standard_normal(E), dtype)
    index = np.argsort(-_np(x) - r.standard_normal(E) * 0.2, axis=1)[:, :k].astype(np.int32)
    index[r.random((T, k)) < 0.05] = -1
    if T:
        index[0, 0] = E + 3 if T > 4 else index[0, 0]        # outside: not counted
    if kw["mask"] is not None:
        kw["mask"] = kw["mask"].reshape(-1)
    return r, seqs, x, index, kw


def _balance_tol(X, index, seqs, sigmoid, spec, dtype, want):
    """Scores: an exponent rounded (2 u |a|), the exponential (2 u), sums over E / 8 and then eight lanes (n u), quotients
    (2 u): (2 |a| + n + 8) u each, of a sigmoid twice that. Their means add u for each token that one lane adds up (at most
    T / 8 of a tile's 4096; tiles are added in 64 bits). slopes are rounded 3 times; the gradient's mean adds E / 8 products."""
    E = X.shape[1]
    s, _ = O.balance_scores(X, sigmoid)
    n = E / 8 + 6
    with np.errstate(all="ignore"):
        a = np.where(s > 0, np.abs(X - X.max(axis=1, keepdims=True)) + (np.abs(X) if sigmoid else 0), 0)
        a = np.minimum(a, 110)
    err = (2 * a + 2 * n + 12) * U * (2 if sigmoid else 1)
    load, counts = spec.get("load"), None
    T, live = sum(len(t) for t in seqs), max(1, sum(len(t) > 0 for t in seqs))
    grad, balance = np.zeros_like(X), 0.0
    top = X.max(axis=1) if T else X[:, :1].max(axis=1, initial=0)
    with np.errstate(all="ignore"):
        lse = top + np.log(np.exp(X - top[:, None]).sum(axis=1))
        soft = np.exp(X - lse[:, None])
    tz = 0.0
    for t in seqs:
        if not len(t):
            continue
        c = np.bincount(index[t][(index[t] >= 0) & (index[t] < E)].reshape(-1), minlength=E) if load is None else load
        f = E * c / max(1, c.sum())
        balance += (f * (s[t] * (err[t] + (len(t) / 8 + 40) * U)).mean(axis=0)).sum() / live
        spread = np.abs(f - 1)
        m = (s[t] * spread).sum(axis=1, keepdims=True)
        grad[t] = abs(spec.get("balance_coef", 0.01)) / (len(t) * live) * s[t] * ((spread + m) * (err[t] + (n + 12) * U)
                                                                                + (s[t] * spread * err[t]).sum(axis=1, keepdims=True))
        if spec.get("z_coef"):
            e = (2 * np.abs(top[t]) + np.abs(lse[t]) * 4 + n + 8) * U
            tz += (2 * np.abs(lse[t]) * e).sum() / T
            grad[t] += abs(spec["z_coef"]) * 2 / T * soft[t] * ((np.abs(lse[t]) * 10 * U + e)[:, None] + np.abs(lse[t])[:, None] * (err[t] + 2 * n * U))
    out = np.array([abs(spec.get("balance_coef", 0.01)) * balance + abs(spec.get("z_coef", 0)) * tz, balance, tz])
    return out, grad * 1.01 + HALF[dtype] * np.abs(want) + 2.0 ** -126


BALANCES = [dict(), dict(z_coef=0.02), dict(balance_coef=0.0, z_coef=1.0), dict(balance_coef=1.0)]


@pytest.mark.parametrize("E,k", [(1, 1), (2, 1), (3, 2), (8, 2), (31, 4), (33, 6), (64, 6), (65, 9), (128, 3), (200, 8), (256, 8), (257, 40),
                                 (512, 64), (1000, 10), (1024, 1)])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_balance_of_every_width(E, k, sigmoid, dtype):
    M = _M()
    for i, (T, S, kind, mask) in enumerate([(1, 1, None, "none"), (33, 1, None, "random"), (300, 7, "part", "random"), (129, 3, None, "empty rows"),
                                            (900, 1, "part", "none"), (31, 70, "whole", "none"), (0, 2, "whole", "none")]):
        spec = BALANCES[(i + E) % len(BALANCES)]
        r, seqs, x, index, kw = _balance_case(i, T, E, k, S, kind, mask, dtype)
        if kind is None:
            kw = {**kw, "sequences": S}
        kw.pop("offsets") if kw["offsets"] is None else None
        load = r.integers(0, 50, E) if i % 3 == 2 else None
        cfg = M.moara_balance_default_config(experts=E, top_k=k, score=M.MOARA_SIGMOID if sigmoid else M.MOARA_SOFTMAX, **spec)
        before = bytes(cfg)
        ix = _gpu(index)
        out, counts, slope = M.moara_balance_loss(cfg, x, ix, load=None if load is None else _gpu(load), **kw)
        gl = torch.full((), -0.6, device="cuda")
        grad = M.moara_balance_loss_backward(cfg, x, slope, gl, **kw)
        assert bytes(cfg) == before and grad.dtype == dtype
        X = _np(x)
        w_out, w_counts, w_grad = O.balance(X, index, seqs, sigmoid, load=load, **spec)
        w_grad = -0.6 * w_grad
        t_out, t_grad = _balance_tol(X, index, seqs, sigmoid, {**spec, "load": load}, dtype, w_grad)
        _close(_np(out), w_out, t_out + 2 * U * np.abs(w_out), f"out {T, S, kind, spec}")
        assert np.array_equal(_np(counts), w_counts)
        _close(_np(grad), w_grad, t_grad, f"gradient {T, S, kind, spec}")
        again = M.moara_balance_loss(cfg, x, ix, load=None if load is None else _gpu(load), **kw)
        assert all(torch.equal(a, b) for a, b in zip(again, (out, counts, slope)))


@pytest.mark.parametrize("T,S,kind", [(8192, 1, None), (8193, 1, None), (20000, 5, "part"), (16384, 16, None), (70000, 300, "whole"),
                                      (40000, 20, "one long")])
def test_balance_of_many_tokens(T, S, kind):
    M = _M()
    for E, k, sigmoid in ((8, 2, False), (64, 6, True), (200, 8, False)):
        r, seqs, x, index, kw = _balance_case(3, T, E, k, S, kind, "random", F32)
        if kind is None:
            kw = {"mask": kw["mask"], "sequences": S}
        spec = dict(z_coef=1e-3)
        cfg = M.moara_balance_default_config(experts=E, top_k=k, score=M.MOARA_SIGMOID if sigmoid else M.MOARA_SOFTMAX, **spec)
        out, counts, slope = M.moara_balance_loss(cfg, x, _gpu(index), **kw)
        grad = M.moara_balance_loss_backward(cfg, x, slope, torch.ones((), device="cuda"), **kw)
        X = _np(x)
        w_out, w_counts, w_grad = O.balance(X, index, seqs, sigmoid, **spec)
        t_out, t_grad = _balance_tol(X, index, seqs, sigmoid, spec, F32, w_grad)
        _close(_np(out), w_out, t_out + 2 * U * np.abs(w_out), "out")
        assert np.array_equal(_np(counts), w_counts)
        _close(_np(grad), w_grad, t_grad, "gradient")


@pytest.mark.parametrize("E", [6, 100])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_balance_of_rows_without_scores(E, sigmoid):
    """Rows that routing gives to no expert, with and without a mask; -inf in some places; scores that underflow."""
    M = _M()
    r = rng(23, E)
    x = r.standard_normal((12, E))
    x[0] = -np.inf
    x[1, 2] = np.nan
    x[2, :4] = -np.inf
    x[3] -= 500
    x[4] += 300
    x[5, 0] = -3e38
    if not sigmoid:
        x[6, 1] = np.inf
    x[7] = np.nan
    index = r.integers(0, E, (12, 2)).astype(np.int32)
    mask = np.ones(12, bool)
    mask[7] = False
    for z in (0.0, 0.1):
        seqs = O.members(12, 1, None, mask)
        cfg = M.moara_balance_default_config(experts=E, top_k=2, score=M.MOARA_SIGMOID if sigmoid else M.MOARA_SOFTMAX, balance_coef=1.0, z_coef=z)
        out, counts, slope = M.moara_balance_loss(cfg, _gpu(x, F32), _gpu(index), mask=_gpu(mask))
        grad = M.moara_balance_loss_backward(cfg, _gpu(x, F32), slope, torch.ones(1, device="cuda"), mask=_gpu(mask))
        X = x.astype(np.float32).astype(float)
        w_out, w_counts, w_grad = O.balance(X, index, seqs, sigmoid, balance_coef=1.0, z_coef=z)
        dead = [0, 1, 7] + ([] if sigmoid else [6])
        assert not grad[dead].any() and np.array_equal(_np(counts), w_counts)
        ok = np.setdiff1d(np.arange(12), dead)
        t_out, t_grad = _balance_tol(X[ok], index[ok], [np.arange(len(ok))], sigmoid, dict(balance_coef=1.0, z_coef=z), F32, w_grad[ok])
        _close(_np(out), w_out, t_out + 2 * U * np.abs(w_out), "out")
        _close(_np(grad)[ok], w_grad[ok], t_grad, "gradient")


def test_balance_of_an_even_load_has_no_gradient():
    M = _M()
    x = torch.randn(64, 16, device="cuda")
    index = torch.arange(64, device="cuda", dtype=torch.int32)[:, None] % 16
    cfg = M.moara_balance_default_config(experts=16, top_k=1, balance_coef=1.0)
    out, _, slope = M.moara_balance_loss(cfg, x, index)
    assert float(out[1]) == pytest.approx(1.0, rel=1e-6)
    assert not M.moara_balance_loss_backward(cfg, x, slope, torch.ones(1, device="cuda")).any()


def test_balance_binding_refusals():
    M = _M()
    cfg = M.moara_balance_default_config(experts=8, top_k=2)
    x, i = torch.zeros(6, 8, device="cuda"), torch.zeros(6, 2, dtype=torch.int32, device="cuda")
    o = torch.tensor([0, 6], device="cuda")
    for a, b, kw in ((x[:, :7], i, {}), (x.half(), i, {}), (x, i.long(), {}), (x, i[:, :1], {}), (x, i, dict(mask=torch.ones(5, dtype=torch.bool, device="cuda"))),
                     (x, i, dict(offsets=o.int())), (x, i, dict(offsets=o, sequences=1)), (x, i, dict(load=torch.zeros(7, dtype=torch.int64, device="cuda"))),
                     (torch.zeros(8, 6, device="cuda").t(), i, {}), (x.cpu(), i, {}), (x, i.cpu(), {})):
        with pytest.raises(ValueError):
            M.moara_balance_loss(cfg, a, b, **kw)
    for kw in (dict(sequences=4), dict(sequences=0), dict(offsets=o[:1])):
        with pytest.raises(M.MoaraError):
            M.moara_balance_loss(cfg, x, i, **kw)


# ---------------------------------------------------------------- streams, graphs, differences, all together

def _policy_inputs(T=300, V=1111, S=6, dtype=BF16):
    r = rng(31, T, V)
    x = _gpu(2 * r.standard_normal((T, V)), dtype)
    lab = _gpu(r.integers(0, V, T))
    lab[::7] = -100
    o = _gpu(np.concatenate([[0], np.sort(r.integers(0, T + 1, S - 1)), [T]]))
    logp = O.token_logps(_np(x), _np(lab))[0]
    old, ref = (_gpu(logp + 0.2 * r.standard_normal(T), F32) for _ in range(2))
    return x, lab, o, old, ref, _gpu(r.standard_normal(S), F32)


def _policy_step(x, lab, o, old, ref, adv):
    M, L = _M(), _L()
    cfg = M.moara_policy_default_config(kl_coef=0.1, entropy_coef=0.02, sequence_advantages=1, reduce=M.MOARA_MEAN_SEQUENCES)
    leaf = x.detach().requires_grad_()
    logp, H = L.token_logps(leaf, lab, temperature=1.25, entropy=True)
    loss, about = L.policy_loss(cfg, logp, adv, old_logp=old, ref_logp=ref, entropy=H, offsets=o, mask=lab >= 0)
    grad, = torch.autograd.grad(loss, leaf)
    return loss.detach(), about, grad


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_policy_step_from_logits_to_their_gradient(dtype):
    x, lab, o, old, ref, adv = _policy_inputs(dtype=dtype)
    loss, about, grad = _policy_step(x, lab, o, old, ref, adv)
    X, labels, scale = _np(x), _np(lab), float(np.float32(0.8))
    seqs = O.members(300, 6, _np(o), labels >= 0)
    per = np.zeros(300)
    for t, a in zip(seqs, _np(adv)):
        per[t] = a

    def forward(y):
        logp, H = O.token_logps(y, labels, scale)
        return O.policy(logp, _np(old), _np(ref), per, H, seqs, kl_coef=0.1, entropy_coef=0.02, reduce="sequences"), logp, H
    (out, _, g, h), logp, H = forward(X)
    np.testing.assert_allclose(_np(about), out, rtol=1e-5, atol=2e-6)
    assert float(loss) == float(about[0])
    want = O.token_logps_grad(X, labels, g, h, scale)
    # log-probabilities off by up to 2^-19 move ratios and distances by as much; the rest as for the gradient alone
    _close(_np(grad), want, _grad_tol(X, labels, np.abs(g) + 1e-12, h, scale, want, dtype) + 2.0 ** -18 * np.abs(want) + 2.0 ** -19 * np.abs(want).max(), "gradient")
    v = rng(33).standard_normal(X.shape)
    e = 1e-5
    slope = (forward(X + e * v)[0][0][0] - forward(X - e * v)[0][0][0]) / (2 * e)
    got = float((_np(grad) * v).sum())
    assert got == pytest.approx(slope, rel=1e-4, abs=2 * HALF[dtype] * float(np.linalg.norm(want)) * 4 + 1e-6)


def test_a_preference_step_in_a_model():
    """Pairs through a linear head and an embedding: gradients of the weights against torch's own in 64 bits."""
    M, L = _M(), _L()
    torch.manual_seed(3)
    V, d, B, T = 97, 16, 6, 12
    emb, head = torch.nn.Embedding(V, d).cuda(), torch.nn.Linear(d, V, bias=False).cuda()
    tokens = torch.randint(0, V, (B, T), device="cuda")
    mask = torch.rand(B, T - 1, device="cuda") < 0.7
    mask[2] = False
    ref = torch.randn(B, T - 1, device="cuda") - 4
    logp = L.token_logps(head(emb(tokens))[:, :-1], tokens[:, 1:])
    loss, rewards, about = L.preference_loss(M.moara_preference_default_config(beta=0.3, smoothing=0.1), logp, ref, mask=mask)
    grads = torch.autograd.grad(3 * loss, [emb.weight, head.weight])
    e64, h64 = emb.weight.detach().cpu().double().requires_grad_(), head.weight.detach().cpu().double().requires_grad_()
    t = tokens.cpu()
    x = e64[t] @ h64.t()
    lp = torch.log_softmax(x[:, :-1], -1).gather(2, t[:, 1:, None])[..., 0]
    D = ((lp - ref.cpu().double()) * mask.cpu()).sum(1)
    z = 0.3 * (D[0::2] - D[1::2])
    want = (0.9 * torch.nn.functional.softplus(-z) + 0.1 * torch.nn.functional.softplus(z)).mean()
    for a, b in zip(grads, torch.autograd.grad(3 * want, [e64, h64])):
        torch.testing.assert_close(a.cpu().double(), b, rtol=1e-4, atol=1e-5)
    assert float(loss.detach()) == pytest.approx(float(want.detach()), rel=1e-5)
    torch.testing.assert_close(rewards.cpu().double(), 0.3 * D, rtol=1e-5, atol=1e-5)


def _every_call(x, lab, o, old, ref, adv):
    """All operators once; their outputs."""
    M = _M()
    logp, H, stats = M.moara_token_logps(x, lab, entropy=True)
    cfg = M.moara_policy_default_config(kl_coef=0.1, entropy_coef=0.02, sequence_advantages=1)
    one = torch.ones(1, device=x.device)
    out, w = M.moara_policy_loss(cfg, logp, adv, old_logp=old, ref_logp=ref, entropy=H, offsets=o)
    g, h = M.moara_policy_loss_backward(cfg, logp, adv, w, one, old_logp=old, ref_logp=ref, entropy=H, offsets=o)
    grad = M.moara_token_logps_backward(x, lab, stats, g, entropy=H, grad_entropy=h)
    pref = M.moara_preference_default_config()
    p_out, rewards, slope = M.moara_preference_loss(pref, logp, ref, offsets=o)
    p_grad = M.moara_preference_loss_backward(pref, logp, slope, one, offsets=o)
    logits = x[:, :40]
    rcfg = M.moara_route_default_config(experts=40, top_k=4)
    index, weight = M.moara_route(rcfg, logits)
    bal = M.moara_balance_default_config(experts=40, top_k=4, z_coef=0.1)
    b_out, counts, b_slope = M.moara_balance_loss(bal, logits, index, offsets=o)
    b_grad = M.moara_balance_loss_backward(bal, logits, b_slope, one, offsets=o)
    return [logp, H, out, g, h, grad, p_out, rewards, p_grad, b_out, counts, b_grad]


@pytest.mark.parametrize("T,S,E", [(40, 4, 8), (6000, 4, 40), (200000, 10, 40), (40000, 1, 256)])
def test_the_loss_by_itself_is_the_first_output(T, S, E):
    """A scalar of its own, the same bits as out[0]; what a caller does to it stays out of the others."""
    M, L = _M(), _L()
    r = np.random.default_rng(T)
    logp, ref = (_gpu(-r.random(T), F32) for _ in range(2))
    o = _gpu(np.linspace(0, T, S + 1).astype(np.int64), torch.int64)
    logits = _gpu(r.normal(size=(T, E)), F32)
    index = M.moara_route(M.moara_route_default_config(experts=E, top_k=2), logits)[0]
    taken = [L.policy_loss(M.moara_policy_default_config(), logp, ref, old_logp=ref, offsets=o),
             L.balance_loss(M.moara_balance_default_config(experts=E, top_k=2, z_coef=0.1), logits, index, offsets=o)]
    if S % 2 == 0:
        taken.append(L.preference_loss(M.moara_preference_default_config(), logp, ref, offsets=o))
    for loss, *_, about in taken:
        assert loss.shape == () and float(loss) != 0 and torch.equal(loss, about[0])
        kept = about.clone()
        loss += 1
        assert torch.equal(about, kept)


def test_losses_on_another_stream():
    M = _M()
    args = _policy_inputs(T=4000, V=700)
    want = _every_call(*args)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = _every_call(*args)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    logp = M.moara_token_logps(args[0], args[1], stream=s)[0]
    also = M.moara_token_logps(args[0], args[1], stream=s.cuda_stream)[0]
    s.synchronize()
    assert torch.equal(logp, want[0]) and torch.equal(also, want[0])


def test_losses_from_two_threads_at_once():
    """Each on its own stream and its own inputs, whose sizes take other kernels: as one call after another."""
    inputs = [_policy_inputs(T=4000, V=700), _policy_inputs(T=300, V=9000, dtype=F32)]
    want = [_every_call(*a) for a in inputs]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(20):
                got = _every_call(*inputs[i])
                s.synchronize()
                wrong.extend((i, n) for n, (a, b) in enumerate(zip(got, want[i])) if not torch.equal(a, b))
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


@pytest.mark.parametrize("T", [300, 9000])
def test_losses_in_captured_graphs(T):
    """Two graphs of the same calls on other inputs, replayed in turn with eager calls between: each replay is as the eager
    call on what the inputs then hold."""
    a, b = _policy_inputs(T=T, V=500), _policy_inputs(T=T, V=640, S=8)
    graphs = []
    for args in (a, b):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            _every_call(*args)
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = _every_call(*args)
        graphs.append((g, args, out))
    for i in range(4):
        for g, args, out in graphs:
            args[0].add_(0.25 * torch.randn_like(args[0]))
            args[5].neg_()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(out, _every_call(*args))), i


def test_a_captured_training_step_with_autograd():
    """Forward and backward of a policy step in one graph, replayed: the eager gradients each time."""
    args = _policy_inputs()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(2):
            _policy_step(*args)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = _policy_step(*args)
    for _ in range(3):
        args[0].mul_(0.9)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, _policy_step(*args)))


# ---------------------------------------------------------------- in the router

@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_a_router_with_a_balance_loss(score):
    from paper_2609_15037_amd.route import ExpertRouter
    M = _M()
    torch.manual_seed(5)
    r = ExpertRouter(24, 12, 3, score=M.MOARA_SIGMOID if score == "sigmoid" else M.MOARA_SOFTMAX).cuda()
    x = torch.randn(150, 24, device="cuda")
    mask = torch.rand(150, device="cuda") < 0.9
    o = torch.tensor([0, 40, 40, 150], device="cuda")
    plain = r(x, mask)
    index, weight, loss = r(x, mask, balance=r.balance_config(balance_coef=0.5, z_coef=0.1), offsets=o)
    assert torch.equal(index, plain[0]) and torch.equal(weight, plain[1])
    grad, = torch.autograd.grad(loss, r.weight)
    W = r.weight.detach().cpu().double().requires_grad_()
    logits = x.cpu().double() @ W.t()
    s = torch.softmax(logits, 1) if score == "softmax" else torch.sigmoid(logits) / torch.sigmoid(logits).sum(1, keepdim=True)
    want, m, ix = 0.0, mask.cpu(), index.cpu().long()
    for a, b in ((0, 40), (40, 150)):
        on = m[a:b]
        f = 12 * torch.bincount(ix[a:b][on].flatten(), minlength=12).double() / (3 * int(on.sum()))
        want = want + 0.5 * (f * s[a:b][on].mean(0)).sum() / 2
    want = want + 0.1 * torch.logsumexp(logits, 1)[m].square().mean()
    assert float(loss.detach()) == pytest.approx(float(want.detach()), rel=1e-5)
    torch.testing.assert_close(grad.cpu().double(), torch.autograd.grad(want, W)[0], rtol=1e-4, atol=1e-6)
    _, _, loss = r(x, balance=r.balance_config(), load=torch.arange(12, device="cuda"))
    loss.backward()


# ---------------------------------------------------------------- the example

def _align():
    import importlib.util
    import os
    from tests.conftest import ROOT
    spec = importlib.util.spec_from_file_location("align_moe", os.path.join(ROOT, "examples", "align_moe.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    return ex


@pytest.mark.parametrize("name", ["preference", "policy"])
def test_the_alignment_example(name):
    """It runs, and the gradients of one of its batches are those of torch's own log-softmax and elementary operations on the
    same model (its products in fp32, whose sums torch may take in any order from pass to pass)."""
    ex = _align()
    about = ex.train(name, steps=6, say=lambda s: print("[align]", s, flush=True))
    assert about.shape == (6, 3 if name == "preference" else 6) and torch.isfinite(about).all()
    torch.manual_seed(1)
    model, reference = ex.Model().cuda(), ex.Model().cuda()
    tokens, answer = ex.batch(6, torch.Generator().manual_seed(2))
    with torch.no_grad():
        old = ex.logps(model, tokens, answer) + 0.1 * torch.randn(answer.shape, device="cuda")
        ref = ex.logps(reference, tokens, answer)
    loss, _ = ex.objective(name, model, reference, old, tokens, answer)
    loss.backward()
    got = {n: None if p.grad is None else p.grad.clone() for n, p in model.named_parameters()}
    model.zero_grad()
    aux = []
    logits = model(tokens, model.layers[0].router.balance_config(balance_coef=1e-2, z_coef=1e-4), aux)
    log = torch.log_softmax(logits[:, :-1].double(), dim=-1)
    logp = torch.where(answer, log.gather(2, tokens[:, 1:, None])[..., 0], 0.0)
    if name == "preference":
        d = (logp - ref).sum(dim=1)
        want = torch.nn.functional.softplus(-0.2 * (d[0::2] - d[1::2])).mean()
    else:
        H = torch.where(answer, -(log.exp() * log).sum(dim=-1), 0.0)
        even = ((tokens[:, 1:] % 2 == 0) & answer).sum(dim=1) / answer.sum(dim=1)
        a = ((even - even.mean()) / (even.std() + 1e-6))[:, None]
        r, q = (logp - old).exp(), ref - logp
        each = -torch.minimum(r * a, r.clamp(0.8, 1.2) * a) + 0.02 * (q.expm1() - q) - 1e-3 * H
        want = (each * answer).sum() / answer.sum()
    want = want + sum(aux)
    assert float(loss.detach()) == pytest.approx(float(want.detach()), rel=1e-4)
    want.backward()
    for n, p in model.named_parameters():
        assert (p.grad is None) == (got[n] is None), n
        if p.grad is not None:
            torch.testing.assert_close(got[n], p.grad, rtol=2e-3, atol=2e-3 * float(p.grad.abs().max()) + 1e-8, msg=n)


def test_the_training_example_with_a_balance_loss():
    import importlib.util
    import os
    from tests.conftest import ROOT
    spec = importlib.util.spec_from_file_location("train_moe", os.path.join(ROOT, "examples", "train_moe.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    losses, share = ex.train(steps=3, balance_loss=0.1, say=lambda s: print("[moe]", s, flush=True))
    assert all(math.isfinite(x) for x in losses) and len(share) == 2


# ---------------------------------------------------------------- calls at the edges

@pytest.mark.parametrize("S", [1, 2, 6, 600, 5000])
@pytest.mark.parametrize("packed", [False, True])
def test_policy_of_no_tokens_needs_no_inputs(S, packed):
    """Sequences without a token: no pointer of an input is needed, that of the sequences' advantages neither; all is 0."""
    import ctypes
    M = _M()
    offsets = torch.zeros(S + 1, dtype=torch.int64, device="cuda") if packed else None
    out, loss, weight = (torch.full((n,), 7.0, device="cuda") for n in (6, 1, S + 1))
    work = torch.full((6 * (S + 130),), math.nan, dtype=torch.float64, device="cuda")
    for whole in (0, 1):
        cfg = M.moara_policy_default_config(sequence_advantages=whole, reduce=whole)
        status = M.lib().moara_policy_loss(ctypes.byref(cfg), None, None, None, None, None, None, 0, offsets.data_ptr() if packed else None,
                                           S, out.data_ptr(), loss.data_ptr(), weight.data_ptr(), work.data_ptr(), None)
        torch.cuda.synchronize()
        assert status == M.MOARA_OK and not out.any() and not loss.any() and not weight.any()
        for t in (out, loss, weight):
            t.fill_(7.0)


def _large(x, T):
    """The tokens of a small case and, from there on, ones whose terms are all 0: of the sizes that take other kernels."""
    y = torch.zeros(1, T, device="cuda")
    y[:, :x.shape[-1]] = x
    return y


@pytest.mark.parametrize("T", [8, 3000, 70001])
@pytest.mark.parametrize("reduce", [0, 1])
def test_policy_of_an_advantage_of_zero(T, reduce):
    """It has no part in the loss and no gradient, also where its ratio overflows, of the tokens' advantages and of a whole
    sequence's; a NaN among its log-probabilities stays one."""
    M = _M()
    logp = _large(torch.tensor([0.0, 0.0, -200.0, 0.5, 100.0]), T)
    old = _large(torch.tensor([-200.0, -math.inf, 0.0, 0.4, 0.0]), T)
    adv = _large(torch.tensor([0.0, -0.0, 0.0, -2.0, 0.0]), T)
    one = torch.ones(1, device="cuda")
    cfg = M.moara_policy_default_config(reduce=reduce)
    out, w = M.moara_policy_loss(cfg, logp, adv, old_logp=old)
    grad, _ = M.moara_policy_loss_backward(cfg, logp, adv, w, one, old_logp=old)
    d = float(logp[0, 3].double() - old[0, 3].double())
    want = 2 * math.exp(d) / T          # one token with a part: its ratio (6 u and |d| u), product, weight, rounding
    assert float(out[0]) == pytest.approx(want, rel=16 * U) and float(out[1]) == float(out[0])
    assert float(grad[0, 3]) == pytest.approx(want, rel=16 * U)
    grad[0, 3] = 0
    assert not grad.any()
    whole = M.moara_policy_default_config(reduce=reduce, sequence_advantages=1)
    out, w = M.moara_policy_loss(whole, logp, torch.zeros(1, device="cuda"), old_logp=old)
    grad, _ = M.moara_policy_loss_backward(whole, logp, torch.zeros(1, device="cuda"), w, one, old_logp=old)
    assert float(out[0]) == 0 and float(out[1]) == 0 and not grad.any()
    logp[0, 1] = math.nan
    out, w = M.moara_policy_loss(cfg, logp, adv, old_logp=old)
    grad, _ = M.moara_policy_loss_backward(cfg, logp, adv, w, one, old_logp=old)
    assert out[0].isnan() and grad[0, 1].isnan() and torch.isfinite(grad[0, [0, 2, 3, 4]]).all()


@pytest.mark.parametrize("T", [8, 3000, 70001])
@pytest.mark.parametrize("kl", ["exp", "linear", "square"])
def test_policy_terms_with_a_coefficient_of_zero(T, kl):
    """Distances and entropies that are only reported leave the loss and the gradients, bit by bit, as they are without."""
    M = _M()
    r = rng(41, T)
    logp, old, adv = (_gpu(r.standard_normal((2, T)), F32) for _ in range(3))
    ref = logp + 0.1
    ref[0, :3] = torch.tensor([150.0, -math.inf, math.inf], device="cuda")
    ref[1, 5] = math.nan
    H = torch.ones(2, T, device="cuda")
    H[1, 2], H[0, 1] = math.inf, math.nan
    one = torch.ones(1, device="cuda")
    cfg = _policy_cfg(M, dict(kl=kl))
    plain, w0 = M.moara_policy_loss(cfg, logp, adv, old_logp=old)
    g0, _ = M.moara_policy_loss_backward(cfg, logp, adv, w0, one, old_logp=old)
    out, w = M.moara_policy_loss(cfg, logp, adv, old_logp=old, ref_logp=ref, entropy=H)
    g, h = M.moara_policy_loss_backward(cfg, logp, adv, w, one, old_logp=old, ref_logp=ref, entropy=H)
    assert torch.isfinite(plain).all() and torch.equal(w, w0)
    assert torch.equal(out[[0, 1, 4, 5]], plain[[0, 1, 4, 5]]) and out[2:4].isnan().all()       # the reports say what there is
    assert torch.equal(g, g0) and not h.any()


def test_preference_of_a_smoothing_of_one():
    """Only the other label's term counts: 0 where the difference is -infinity."""
    M = _M()
    logp = torch.tensor([[-math.inf, -1.0], [-1.0, -1.0], [-1.0, -2.0], [-1.5, -2.0]], device="cuda")
    cfg = M.moara_preference_default_config(beta=0.5, smoothing=1.0)
    out, rewards, slope = M.moara_preference_loss(cfg, logp)
    z = 0.5 * 0.5
    assert float(out[0]) == pytest.approx(math.log1p(math.exp(z)) / 2, rel=4 * U)
    grad = M.moara_preference_loss_backward(cfg, logp, slope, torch.ones(1, device="cuda"))
    s = 0.5 / (1 + math.exp(-z)) / 2
    np.testing.assert_allclose(_np(grad), [[0, 0], [0, 0], [s, s], [-s, -s]], rtol=8 * U)


@pytest.mark.parametrize("T,S", [(1000, 4), (3000, 64), (100000, 300), (100000, 4)])
@pytest.mark.parametrize("seed", range(3))
def test_falling_offsets_give_the_same_sums_each_time(T, S, seed):
    """Whatever the workspace held: sums of tokens, the same bits each time."""
    import ctypes
    M = _M()
    r = rng(43, seed, T, S)
    offsets = _gpu(r.integers(-5, T + 5, S + 1))
    logp = _gpu(-r.exponential(size=T), F32)
    pre, pol = M.moara_preference_default_config(kind=M.MOARA_PREF_SQUARE, beta=1.0), M.moara_policy_default_config()
    found = []
    for fill in (0.0, math.nan, 1e300):
        work = torch.full((6 * (S + T // 512 + 130),), fill, dtype=torch.float64, device="cuda")
        out, rewards, slope, about, weight = (torch.full((n,), 5.0, device="cuda") for n in (3, S, S + 1, 6, S + 1))
        assert M.lib().moara_preference_loss(ctypes.byref(pre), logp.data_ptr(), None, None, T, offsets.data_ptr(), S, out.data_ptr(), None,
                                             rewards.data_ptr(), slope.data_ptr(), work.data_ptr(), None) == M.MOARA_OK
        work.fill_(fill)
        assert M.lib().moara_policy_loss(ctypes.byref(pol), logp.data_ptr(), None, None, None, logp.data_ptr(), None, T, offsets.data_ptr(),
                                         S, about.data_ptr(), None, weight.data_ptr(), work.data_ptr(), None) == M.MOARA_OK
        torch.cuda.synchronize()
        found.append(torch.cat([out, rewards, slope, about, weight]))
        total = float(logp.double().sum())
        assert torch.isfinite(found[-1]).all() and (rewards <= 0).all() and (rewards >= total * S).all()
    assert torch.equal(found[0], found[1]) and torch.equal(found[0], found[2])


@pytest.mark.parametrize("kind", [torch.int64, torch.int32, torch.uint8, torch.bool])
def test_losses_of_masks_beside_views(kind):
    """A tokenizer's mask without its first position, and int32 offsets: as the library's own types, gradients too."""
    M, L = _M(), _L()
    r = rng(47)
    whole = _gpu((r.random((6, 41)) < 0.7).astype(np.int64)).to(kind)
    logp, ref, adv = (_gpu(-r.exponential(size=(6, 40)), F32) for _ in range(3))
    pre, pol = M.moara_preference_default_config(), M.moara_policy_default_config()
    o = _gpu(np.array([0, 40, 41, 90, 240]))
    found = []
    for mask, offsets in ((whole[:, 1:], o.int()), ((whole[:, 1:] != 0).contiguous(), o)):
        x = logp.clone().requires_grad_()
        flat = dict(offsets=offsets, mask=mask.reshape(-1))
        losses = [L.preference_loss(pre, x, ref, mask=mask)[0], L.policy_loss(pol, x, adv, ref, mask=mask)[0],
                  L.preference_loss(pre, x.view(-1), **flat)[0], L.policy_loss(pol, x.view(-1), adv.view(-1), **flat)[0]]
        found.append([loss.detach() for loss in losses] + [torch.autograd.grad(loss, x)[0] for loss in losses])
    assert all(torch.equal(a, b) and a.any() for a, b in zip(*found))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("MiB", [200, 340])
@pytest.mark.parametrize("gap", [0, 3])
def test_logps_past_the_caches(dtype, MiB, gap):
    """Sizes whose gradients, and whose logits too, are read and written past the caches, and the vocabularies that narrow and
    wide rows take; a few rows with a label, all others' gradients 0 and as many as there are."""
    M = _M()
    for V in (300, 3001, 40000):
        T = (MiB << 20) // (V * (4 if dtype == F32 else 2))
        x = torch.zeros(T, V + gap, dtype=dtype, device="cuda")[:, :V]
        rows = torch.tensor([0, 1, T // 2, T - 1], device="cuda")
        small, lab_small, g_small, h_small = _case(V, 4, V, dtype)
        lab_small[2:] = torch.tensor([V // 2, V - 1], device="cuda")
        x[rows] = small
        lab, g, h = torch.full((T,), -100, device="cuda"), torch.ones(T, device="cuda"), torch.ones(T, device="cuda")
        lab[rows], g[rows], h[rows] = lab_small, g_small + 0.5, h_small - 0.5
        X, labels, gn, hn = _np(small), _np(lab_small), _np(g[rows]), _np(h[rows])
        want, wantH = O.token_logps(X, labels)
        tol, tolH, _ = _logps_tol(X, labels, 1.0)       # as few rows add up: on 16, 64 and at least 256 lanes
        for entropy in (False, True):
            logp, H, stats = M.moara_token_logps(x, lab, entropy=entropy)
            _close(_np(logp[rows]), want, tol, "logp")
            assert int(logp.count_nonzero()) <= 4
            if entropy:
                _close(_np(H[rows]), wantH, tolH, "entropy")
                assert int(H.count_nonzero()) <= 4
            grad = M.moara_token_logps_backward(x, lab, stats, g, entropy=H, grad_entropy=h if entropy else None)
            ref = O.token_logps_grad(X, labels, gn, hn if entropy else None)
            _close(_np(grad[rows]), ref, _grad_tol(X, labels, gn, hn if entropy else None, 1.0, ref, dtype), "gradient")
            grad[rows] = 0
            assert not grad.any()


@pytest.mark.parametrize("E,T,S", [(256, 40000, 1), (1000, 9000, 1), (256, 70000, 2)])
def test_balance_of_many_cells_with_another_load(E, T, S):
    """Cells that are added up by columns first, with counts given for f: this call's counts stay its own."""
    M = _M()
    r, seqs, x, index, kw = _balance_case(53, T, E, 4, S, None, "random", F32)
    load = r.integers(0, 900, E)
    cfg = M.moara_balance_default_config(experts=E, top_k=4, z_coef=1e-3)
    kw = dict(mask=kw["mask"], sequences=S)
    out, counts, slope = M.moara_balance_loss(cfg, x, _gpu(index), load=_gpu(load), **kw)
    grad = M.moara_balance_loss_backward(cfg, x, slope, torch.ones((), device="cuda"), **kw)
    X, spec = _np(x), dict(z_coef=1e-3)
    w_out, w_counts, w_grad = O.balance(X, index, seqs, False, load=load, **spec)
    t_out, t_grad = _balance_tol(X, index, seqs, False, {**spec, "load": load}, F32, w_grad)
    _close(_np(out), w_out, t_out + 2 * U * np.abs(w_out), "out")
    assert np.array_equal(_np(counts), w_counts)
    _close(_np(grad), w_grad, t_grad, "gradient")


def test_losses_from_two_threads_all_return():
    """As test_losses_from_two_threads_at_once, counting the calls that came back: an error in a thread fails too."""
    inputs = [_policy_inputs(T=4000, V=700), _policy_inputs(T=300, V=9000, dtype=F32)]
    want = [_every_call(*a) for a in inputs]
    torch.cuda.synchronize()
    same = [0, 0]

    def work(i):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(10):
                got = _every_call(*inputs[i])
                s.synchronize()
                same[i] += all(torch.equal(a, b) for a, b in zip(got, want[i]))
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert same == [10, 10]
