"""The losses without a GPU: refusals of the C ABI before anything is enqueued, the oracle against hand-written values and
differences, the partition of packed tokens into cells, the autograd wrappers with stand-ins for the library's calls."""
import ctypes
import math
import os

import numpy as np
import pytest

from oracle import loss_oracle as O

M = pytest.importorskip("paper_2609_15037_amd.moara")
torch = pytest.importorskip("torch")
from paper_2609_15037_amd import losses as L  # noqa: E402

P = 1 << 20         # an address that no refused call may touch
ARG, SHAPE, UNS = M.MOARA_E_ARG, M.MOARA_E_SHAPE, M.MOARA_E_UNSUPPORTED


@pytest.fixture
def lib():
    if not os.path.exists(M.LIB_PATH):
        pytest.skip("libmoara.so not built")
    return M.lib()


# ---------------------------------------------------------------- refusals

LOGITS = dict(logits=P, dtype=0, tokens=4, vocab=10, row=10, inner=4, outer=0, scale=1.0, labels=P)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), ARG), (dict(tokens=-1), SHAPE), (dict(tokens=(1 << 40) + 1), SHAPE), (dict(vocab=0), SHAPE),
    (dict(vocab=(1 << 30) + 1), SHAPE), (dict(scale=0.0), ARG), (dict(scale=-1.0), ARG), (dict(scale=math.nan), ARG),
    (dict(scale=math.inf), ARG), (dict(scale=3e38), ARG), (dict(row=9), SHAPE), (dict(row=0), SHAPE), (dict(row=-10), SHAPE), (dict(inner=0), SHAPE),
    (dict(inner=2, outer=9), SHAPE), (dict(inner=2, outer=0), SHAPE), (dict(inner=2, outer=1 << 45), SHAPE),
    (dict(row=1 << 45), SHAPE), (dict(logits=None), ARG), (dict(labels=None), ARG),
    (dict(logits=P + 2), ARG), (dict(logits=P + 1, dtype=1), ARG), (dict(labels=P + 4), ARG),
    (dict(inner=(1 << 40) - 1, tokens=1 << 40, row=1 << 40, outer=1 << 62), SHAPE)])
def test_logits_are_refused(lib, kw, status):
    a = tuple({**LOGITS, **kw}.values())
    assert lib.moara_token_logps(*a, P, None, P, None) == status
    assert lib.moara_token_logps_backward(*a, P, P, None, None, P, 1 << 40, None) == status
    assert M.moara_last_error()


def test_logps_outputs_are_refused(lib):
    a = tuple(LOGITS.values())
    for o in ((None, None, P), (P, None, None), (P + 2, None, P), (P, P + 1, P), (P, None, P + 8)):
        assert lib.moara_token_logps(*a, *o, None) == ARG, o
    for o in ((None, P, None, None, P, 10), (P, None, None, None, P, 10), (P, P, None, None, None, 10), (P, P, None, P, P, 10),
              (P + 8, P, None, None, P, 10), (P, P + 1, None, None, P, 10), (P, P, P + 2, P, P, 10), (P, P, P, P + 2, P, 10),
              (P, P, None, None, P + 2, 10)):
        assert lib.moara_token_logps_backward(*a, *o, None) == ARG, o
    assert lib.moara_token_logps_backward(*a, P, P, None, None, P, 9, None) == SHAPE
    none = tuple({**LOGITS, "tokens": 0, "logits": None, "labels": None}.values())
    assert lib.moara_token_logps(*none, None, None, None, None) == M.MOARA_OK           # nothing to do
    assert lib.moara_token_logps_backward(*none, None, None, None, None, None, 10, None) == M.MOARA_OK


PACKED = [(dict(tokens=-1), SHAPE), (dict(tokens=(1 << 33) + 1, sequences=1), SHAPE), (dict(sequences=0), SHAPE),
          (dict(sequences=-2), SHAPE), (dict(sequences=(1 << 21) + 2), SHAPE), (dict(tokens=9), SHAPE), (dict(offsets=P + 4), ARG)]


@pytest.mark.parametrize("kw,status", PACKED + [
    (dict(sequences=3, tokens=9), SHAPE), (dict(logp=None), ARG), (dict(logp=P + 1), ARG), (dict(ref=P + 2), ARG),
    (dict(out=None), ARG), (dict(loss=P + 2), ARG), (dict(rewards=None), ARG), (dict(slope=None), ARG), (dict(work=None, tokens=8000), ARG), (dict(work=P + 4), ARG),
    (dict(beta=0.0), ARG), (dict(beta=-1.0), ARG), (dict(beta=math.inf), ARG), (dict(margin=math.nan), ARG), (dict(kind=3), ARG),
    (dict(kind=-1), ARG), (dict(smoothing=1.5), ARG), (dict(smoothing=-0.1), ARG), (dict(smoothing=0.1, kind=1), ARG),
    (dict(margin=0.5, kind=2), ARG)])
def test_preference_calls_are_refused(lib, kw, status):
    cfg = M.moara_preference_default_config(**{k: v for k, v in kw.items() if k in ("beta", "margin", "smoothing", "kind")})
    a = {**dict(logp=P, ref=None, mask=None, tokens=8, offsets=None, sequences=4, out=P, loss=None, rewards=P, slope=P, work=P), **kw}
    call = [a[k] for k in ("logp", "ref", "mask", "tokens", "offsets", "sequences", "out", "loss", "rewards", "slope", "work")]
    assert lib.moara_preference_loss(ctypes.byref(cfg), *call, None) == status
    if (kw, status) in PACKED:
        assert lib.moara_preference_loss_backward(P, P, None, a["tokens"], a["offsets"], a["sequences"], P, None) == status


def test_preference_backward_arguments_are_refused(lib):
    for a in ((None, P, P), (P, None, P), (P, P, None), (P + 1, P, P), (P, P + 2, P), (P, P, P + 2)):
        assert lib.moara_preference_loss_backward(a[0], a[1], None, 8, None, 4, a[2], None) == ARG, a
    assert lib.moara_preference_loss_backward(P, P, None, 9, None, 3, P, None) == SHAPE
    assert lib.moara_preference_loss(None, P, None, None, 8, None, 4, P, None, P, P, P, None) == ARG


@pytest.mark.parametrize("kw,status", PACKED + [
    (dict(logp=None), ARG), (dict(adv=None), ARG), (dict(logp=P + 1), ARG), (dict(old=P + 2), ARG), (dict(ref=P + 2), ARG),
    (dict(adv=P + 2), ARG), (dict(entropy=P + 2), ARG), (dict(out=None), ARG), (dict(loss=P + 2), ARG), (dict(weight=None), ARG), (dict(work=None, tokens=8000), ARG),
    (dict(work=P + 4), ARG), (dict(clip_low=-0.1), ARG), (dict(clip_low=1.1), ARG), (dict(clip_high=-0.1), ARG),
    (dict(clip_high=math.nan), ARG), (dict(kl_coef=0.1, ref=None), ARG), (dict(entropy_coef=0.1, entropy=None), ARG),
    (dict(kl_coef=math.inf), ARG), (dict(entropy_coef=math.nan), ARG), (dict(divisor=-1.0), ARG), (dict(divisor=math.inf), ARG),
    (dict(kl=3), ARG), (dict(reduce=2), ARG)])
def test_policy_calls_are_refused(lib, kw, status):
    names = [n for n, _ in M.moara_policy_config._fields_]
    cfg = M.moara_policy_default_config(**{k: v for k, v in kw.items() if k in names})
    a = {**dict(logp=P, old=P, ref=P, entropy=P, adv=P, mask=None, tokens=8, offsets=None, sequences=4, out=P, loss=None, weight=P,
           work=P), **kw}
    order = ("logp", "old", "ref", "entropy", "adv", "mask", "tokens", "offsets", "sequences", "out", "loss", "weight", "work")
    assert lib.moara_policy_loss(ctypes.byref(cfg), *[a[k] for k in order], None) == status
    if not {"entropy", "entropy_coef", "out", "loss", "weight", "work"} & set(kw) or kw.get("entropy_coef") != kw.get("entropy_coef"):
        back = [a[k] for k in ("logp", "old", "ref", "adv", "mask", "tokens", "offsets", "sequences")]
        assert lib.moara_policy_loss_backward(ctypes.byref(cfg), *back, P, P, P, None, None) == status
    assert lib.moara_policy_loss(None, *[a[k] for k in order], None) == ARG


def test_policy_backward_arguments_are_refused(lib):
    cfg = ctypes.byref(M.moara_policy_default_config())
    for a in ((None, P, P, None), (P, None, P, None), (P, P, None, None), (P + 1, P, P, None), (P, P + 2, P, None),
              (P, P, P + 2, None), (P, P, P, P + 2)):
        assert lib.moara_policy_loss_backward(cfg, P, None, None, P, None, 8, None, 4, *a, None) == ARG, a


@pytest.mark.parametrize("kw,status", PACKED + [
    (dict(experts=0), ARG), (dict(top_k=0), ARG), (dict(score=2), ARG), (dict(logits_dtype=2), ARG),
    (dict(balance_coef=math.nan), ARG), (dict(z_coef=math.inf), ARG), (dict(experts=1025, row=1025), UNS), (dict(top_k=65), UNS),
    (dict(logits=None), ARG), (dict(logits=P + 2), ARG), (dict(row=63), SHAPE), (dict(index=None), ARG), (dict(index=P + 2), ARG),
    (dict(load=P + 4), ARG), (dict(out=None), ARG), (dict(loss=P + 2), ARG), (dict(counts=None), ARG), (dict(counts=P + 4), ARG), (dict(slope=None), ARG),
    (dict(work=None), ARG), (dict(work=P + 4), ARG)])
def test_balance_calls_are_refused(lib, kw, status):
    names = [n for n, _ in M.moara_balance_config._fields_]
    cfg = M.moara_balance_default_config(**{k: v for k, v in kw.items() if k in names})
    a = {**dict(logits=P, tokens=8, row=64, index=P, mask=None, offsets=None, sequences=4, load=None, out=P, loss=None, counts=P,
                slope=P, work=P), **kw}
    order = ("logits", "tokens", "row", "index", "mask", "offsets", "sequences", "load", "out", "loss", "counts", "slope", "work")
    assert lib.moara_balance_loss(ctypes.byref(cfg), *[a[k] for k in order], None) == status
    if not {"index", "load", "out", "loss", "counts", "slope", "work"} & set(kw):
        back = [a[k] for k in ("logits", "tokens", "row", "mask", "offsets", "sequences")]
        assert lib.moara_balance_loss_backward(ctypes.byref(cfg), *back, P, P, P, None) == status
    assert lib.moara_balance_loss(None, *[a[k] for k in order], None) == ARG


def test_balance_backward_arguments_are_refused(lib):
    cfg = ctypes.byref(M.moara_balance_default_config())
    for a in ((None, P, P), (P, None, P), (P, P, None), (P + 1, P, P), (P, P + 2, P), (P, P, P + 2)):
        assert lib.moara_balance_loss_backward(cfg, P, 8, 64, None, None, 4, *a, None) == ARG, a


def test_default_configurations_need_a_place(lib):
    for f in ("preference", "policy", "balance"):
        assert getattr(lib, f"moara_{f}_default_config")(None) == ARG


def test_tensors_on_the_host_are_refused():
    """The binding takes GPU tensors only, and says which one is not."""
    x, lab = torch.zeros(3, 5), torch.zeros(3, dtype=torch.int64)
    for call in (lambda: M.moara_token_logps(x, lab), lambda: M.moara_preference_loss(None, x),
                 lambda: M.moara_policy_loss(M.moara_policy_config(), x, x),
                 lambda: M.moara_balance_loss(M.moara_balance_config(experts=5, top_k=1), x, lab)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


@pytest.mark.parametrize("shape,strides,want", [
    ((4, 10), (10, 1), (4, 10, 10, 4, 0)), ((4, 10), (16, 1), (4, 10, 16, 4, 0)), ((1, 10), (7, 1), (1, 10, 10, 1, 0)),
    ((3, 5, 10), (60, 10, 1), (15, 10, 10, 5, 60)), ((3, 5, 10), (50, 10, 1), (15, 10, 10, 5, 50)),
    ((1, 5, 10), (999, 12, 1), (5, 10, 12, 5, 0)), ((3, 1, 10), (60, 10, 1), (3, 10, 60, 3, 0)),
    ((0, 10), (10, 1), (0, 10, 10, 1, 0)), ((0, 5, 10), (50, 10, 1), (0, 10, 10, 5, 0)), ((3, 0, 10), (10, 10, 1), (0, 10, 10, 1, 10)),
    ((4, 1), (1, 1), (4, 1, 1, 4, 0)), ((4, 1), (3, 3), (4, 1, 3, 4, 0))])
def test_rows_of_logits(monkeypatch, shape, strides, want):
    monkeypatch.setattr(M, "_on_gpu", lambda t, device, what: 0)
    n = 1 + sum(max(a - 1, 0) * s for a, s in zip(shape, strides))
    t = torch.zeros(max(n, 1)).as_strided(shape, strides)
    dev, dtype, *rest = M._logits_rows(t)
    assert (dev, dtype) == (0, M.MOARA_F32) and tuple(rest) == want
    tokens, vocab, ld, inner, outer = rest
    at = [(r // inner) * outer + (r % inner) * ld for r in range(tokens)]      # where the library looks for row r
    flat = t.reshape(-1, shape[-1])
    base = torch.arange(max(n, 1), dtype=torch.float32)
    assert [int(x) for x in base.as_strided(shape, strides).reshape(-1, shape[-1])[:, 0]] == at or not flat.numel()


def test_rows_without_unit_stride_are_refused(monkeypatch):
    monkeypatch.setattr(M, "_on_gpu", lambda t, device, what: 0)
    for t in (torch.zeros(10, 4).t(), torch.zeros(5), torch.zeros(2, 2, 2, 5), torch.zeros(4, 0)):
        with pytest.raises(ValueError):
            M._logits_rows(t)


def test_overlapping_outputs_are_seen():
    x = torch.zeros(100)
    a, b, c = x[:40].view(4, 10), x[40:80].view(4, 10), x[39:79].view(4, 10)
    assert not M._overlap(a, b) and M._overlap(a, c) and M._overlap(b, c) and not M._overlap(a, x[:0])


# ---------------------------------------------------------------- cells of packed tokens

def _cells(offsets, tokens, tile):
    """The kernels' partition, step by step as they take it: for each cell its sequence, its tokens and those to clear."""
    S = len(offsets) - 1
    first = lambda s: min(max(int(offsets[s]), 0), tokens)  # noqa: E731
    out = []
    for i in range(S + -(-tokens // tile) - 1):
        lo, hi = -1, S
        while hi - lo > 1:
            step = (hi - lo + 62) // 64
            n = sum(lo + 1 + l * step < hi and (lo + 1 + l * step) + first(lo + 1 + l * step) // tile <= i for l in range(64))
            nxt = lo + 1 + n * step
            lo, hi = (nxt - step if n else lo), min(nxt, hi)
        s, at = lo, i - max(lo, 0)
        t0 = at * tile
        t1 = min(t0 + tile, tokens)
        b = first(max(s, 0))
        if s < 0:
            out.append((s, (0, 0), [(t0, min(b, t1))]))
            continue
        e = max(first(s + 1), b)
        clear = [(t0, b)] if s == 0 and at == b // tile else []
        clear += [(max(e, t0), t1)] if s == S - 1 else []
        out.append((s, (max(b, t0), min(e, t1)), clear))
    return out


@pytest.mark.parametrize("seed", range(40))
def test_cells_partition_the_tokens(seed):
    g = np.random.default_rng(seed)
    tile = int(g.choice([1, 4, 32]))
    tokens, S = int(g.integers(0, 400)), int(g.choice([1, 2, 3, 63, 64, 65, 130, 300]))
    a, b = sorted(g.integers(0, tokens + 1, 2)) if seed % 3 else (0, tokens)
    offsets = np.concatenate([[a], np.sort(g.integers(a, b + 1, S - 1)), [b]])
    if seed % 4 == 0 and tile > 1:
        offsets = offsets // tile * tile            # every bound on a tile's
    owner = np.full(tokens, -2)
    sums = {}
    for i, (s, (x, y), clear) in enumerate(_cells(offsets, tokens, tile)):
        for k, (u, v) in [(s, (x, y))] + [(-1, c) for c in clear]:
            if v > u:
                assert 0 <= u and v <= tokens and (owner[u:v] == -2).all()
                owner[u:v] = k
        if y > x:
            sums.setdefault(s, []).append(i)
    want = np.full(tokens, -1)
    for s in range(S):
        want[offsets[s]:offsets[s + 1]] = s
    assert (owner == want).all()
    for s in range(S):                              # the cells that a sequence's sum reads
        x, y = offsets[s], offsets[s + 1]
        first = s + x // tile
        last = s + (y - 1) // tile + 1 if y > x else first
        assert list(range(first, last)) == sums.get(s, [])


@pytest.mark.parametrize("seed", range(30))
def test_cells_of_falling_offsets_stay_inside(seed):
    g = np.random.default_rng(1000 + seed)
    tokens, S, tile = int(g.integers(0, 300)), int(g.choice([1, 2, 65, 200])), int(g.choice([1, 32]))
    offsets = g.integers(-2 ** 62, 2 ** 62, S + 1) if seed % 2 else g.integers(-5, tokens + 6, S + 1)
    cells = _cells(offsets, tokens, tile)
    for s, own, clear in cells:
        assert -1 <= s < S
        for u, v in [own] + clear:
            assert v <= u or (0 <= u and v <= tokens)
    for s in range(S):
        x, y = (min(max(int(o), 0), tokens) for o in offsets[s:s + 2])
        assert not y > x or s + (y - 1) // tile < len(cells)


# ---------------------------------------------------------------- the oracle

def test_oracle_of_known_values():
    x = np.log(np.array([[1.0, 2.0, 5.0], [1.0, 1.0, 2.0], [3.0, 3.0, 2.0]]))
    lab = np.array([2, 0, -100])
    lp, H = O.token_logps(x, lab)
    np.testing.assert_allclose(lp, [math.log(5 / 8), math.log(1 / 4), 0])
    np.testing.assert_allclose(H[:2], [-(1 / 8 * math.log(1 / 8) + 1 / 4 * math.log(1 / 4) + 5 / 8 * math.log(5 / 8)), 1.5 * math.log(2)])
    assert H[2] == 0
    g = O.token_logps_grad(x, lab, np.array([1.0, 2.0, 3.0]))
    np.testing.assert_allclose(g, [[-1 / 8, -2 / 8, 3 / 8], [1.5, -0.5, -1.0], [0, 0, 0]])
    np.testing.assert_allclose(O.token_logps(x, lab, 2.0)[0][0], math.log(25 / 30))
    # pairs: sums 3 - 1 = 2 and -1 - 2 = -3; z = 1 and -1.5
    logp = np.array([1.0, 2.0, 1.0, -1.0, 2.0])
    seqs = O.members(5, 4, [0, 2, 3, 4, 5])
    out, rewards, grad = O.preference(logp, None, seqs, beta=0.5)
    np.testing.assert_allclose(out, [(math.log1p(math.exp(-1)) + math.log1p(math.exp(1.5))) / 2, 0.5, -0.25])
    np.testing.assert_allclose(rewards, [1.5, 0.5, -0.5, 1.0])
    s = [0.25 / (1 + math.exp(1)), 0.25 / (1 + math.exp(-1.5))]
    np.testing.assert_allclose(grad, [-s[0], -s[0], s[0], -s[1], s[1]])
    out, _, grad = O.preference(logp, None, seqs, kind="hinge", beta=0.25, average=True)
    np.testing.assert_allclose(out, [((1 - 0.125) + (1 + 0.75)) / 2, 0.5, (0.125 - 0.75) / 2])
    np.testing.assert_allclose(grad, [-0.0625, -0.0625, 0.125, -0.125, 0.125])
    out, _, grad = O.preference(logp, np.zeros(5), seqs, kind="square", beta=0.5)
    np.testing.assert_allclose(out[0], (1 + 16) / 2)
    np.testing.assert_allclose(grad, [1, 1, -1, -4, 4])
    # ratios 1.5 (clipped for A > 0, not for A < 0), 0.5 (the other way round)
    d = np.log(np.array([1.5, 1.5, 0.5, 0.5]))
    a = np.array([1.0, -1.0, 1.0, -1.0])
    out, w, grad, ge = O.policy(d, np.zeros(4), None, a, np.ones(4), O.members(4, 2), entropy_coef=0.1)
    np.testing.assert_allclose(out[1:5], [-(1.2 - 1.5 + 0.5 - 0.8) / 4, 0, 1, 0.5])
    np.testing.assert_allclose(out[0], out[1] - 0.1)
    np.testing.assert_allclose(grad, [0, 1.5 / 4, -0.5 / 4, 0])
    np.testing.assert_allclose(ge, -0.025)
    out, w, grad, _ = O.policy(np.zeros(3), None, np.log([2.0, 1.0, 0.5]), np.zeros(3), None, O.members(3, 2, [0, 1, 3]), kl_coef=1.0,
                               reduce="sequences")
    np.testing.assert_allclose(w, [0.5, 0.25])
    np.testing.assert_allclose(out[2], 0.5 * (1 - math.log(2)) + 0.25 * (math.log(2) - 0.5))
    np.testing.assert_allclose(grad, [-0.5, 0, 0.125])
    # two experts: load (3, 1) of 4, mean scores (0.7, 0.3): 1.5 0.7 + 0.5 0.3
    x = np.log(np.array([[0.9, 0.1], [0.5, 0.5]]))
    out, c, _ = O.balance(x, np.array([[0, 0], [0, 1]]), O.members(2, 1), balance_coef=0.1, z_coef=1.0)
    np.testing.assert_allclose(out, [0.12, 1.2, 0], atol=1e-15)
    assert c.tolist() == [[3, 1]]
    out, c, _ = O.balance(x + 1, np.array([[0, -1], [1, 7]]), O.members(2, 2), balance_coef=1.0, z_coef=1.0)
    np.testing.assert_allclose(out, [(1.8 + 1.0) / 2 + 1, 1.4, 1])
    assert c.tolist() == [[1, 0], [0, 1]]


def _difference(f, x, v, h=1e-5):
    return (f(x + h * v) - f(x - h * v)) / (2 * h)


@pytest.mark.parametrize("seed", range(6))
def test_oracle_gradients_are_differences(seed):
    """Central differences of smooth functions: an error of h^2 times the third derivative, and of rounding over h."""
    g = np.random.default_rng(seed)
    close = dict(rtol=1e-5, atol=1e-8)
    x, lab, a, b = g.normal(size=(5, 9)), g.integers(-1, 10, 5), g.normal(size=5), g.normal(size=5)
    f = lambda x: (O.token_logps(x, lab, 1.3)[0] * a).sum() + (O.token_logps(x, lab, 1.3)[1] * b).sum()  # noqa: E731
    v = g.normal(size=x.shape)
    np.testing.assert_allclose((O.token_logps_grad(x, lab, a, b, 1.3) * v).sum(), _difference(f, x, v), **close)
    T, S = 40, 8
    off = np.concatenate([[2], np.sort(g.integers(2, 38, S - 1)), [38]])
    seqs = O.members(T, S, off, g.random(T) < 0.7)
    lp, ref, old, v = (g.normal(size=T) for _ in range(4))
    for kw in (dict(smoothing=0.1, margin=0.3), dict(average=True), dict(kind="hinge", beta=0.05), dict(kind="square", beta=0.4)):
        np.testing.assert_allclose((O.preference(lp, ref, seqs, **kw)[2] * v).sum(),
                                   _difference(lambda y: O.preference(y, ref, seqs, **kw)[0][0], lp, v), **close)
    adv, ent = g.normal(size=T), g.random(T)
    for kw in (dict(kl="exp", kl_coef=0.3), dict(kl="linear", kl_coef=0.3, reduce="sequences"),
               dict(kl="square", kl_coef=0.2, divisor=7.0, entropy_coef=0.1)):
        out = O.policy(lp, old, ref, adv, ent, seqs, **kw)
        np.testing.assert_allclose((out[2] * v).sum(), _difference(lambda y: O.policy(y, old, ref, adv, ent, seqs, **kw)[0][0], lp, v), **close)
        np.testing.assert_allclose((out[3] * v).sum(), _difference(lambda y: O.policy(lp, old, ref, adv, y, seqs, **kw)[0][0], ent, v), **close)
    E = 7
    x, v = g.normal(size=(T, E)), g.normal(size=(T, E))
    index = g.integers(-1, E, (T, 2))
    for kw in (dict(), dict(z_coef=0.1), dict(sigmoid=True, z_coef=0.1), dict(sigmoid=True, load=g.integers(0, 9, E))):
        np.testing.assert_allclose((O.balance(x, index, seqs, **kw)[2] * v).sum(),
                                   _difference(lambda y: O.balance(y, index, seqs, **kw)[0][0], x, v), **close)


@pytest.mark.parametrize("plant", ["label_shifted", "no_log_in_entropy", "rejected_first", "clip_both_sides", "token_mean", "bias_counted"])
def test_oracle_pins_catch_planted_mistakes(plant, monkeypatch):
    if plant == "label_shifted":
        real = O.token_logps
        monkeypatch.setattr(O, "token_logps", lambda x, lab, scale=1.0: real(x, np.where(lab > 0, lab - 1, lab), scale))
    elif plant == "no_log_in_entropy":
        monkeypatch.setattr(O, "xlogy", lambda p, log: p)
    elif plant == "rejected_first":
        real_p = O.preference_pair
        monkeypatch.setattr(O, "preference_pair", lambda h, *a: real_p(-h, *a))
    elif plant == "clip_both_sides":
        real_t = O.policy_terms

        def both(logp, old, ref, adv, low, high, kl="exp"):
            gain, slope, *rest = real_t(logp, old, ref, adv, low, high, kl)
            return np.clip(np.exp(logp - (0 if old is None else old)), 1 - low, 1 + high) * adv, slope, *rest
        monkeypatch.setattr(O, "policy_terms", both)
    elif plant == "token_mean":
        real_w = O.policy_weights
        monkeypatch.setattr(O, "policy_weights", lambda seqs, reduce="tokens", divisor=0.0: real_w(seqs, "tokens", divisor))
    else:
        real_s = O.balance_scores
        monkeypatch.setattr(O, "balance_scores", lambda x, sigmoid: (real_s(x, sigmoid)[0] + 0.1, real_s(x, sigmoid)[1]))
    with pytest.raises(AssertionError):
        test_oracle_of_known_values()


# ---------------------------------------------------------------- autograd wrappers

@pytest.fixture
def calls(monkeypatch):
    """The library's calls replaced by recorders that answer with tensors of the right shapes."""
    seen = []

    def record(name, answer):
        def f(*a, **kw):
            seen.append((name, a, kw))
            return answer(*a, **kw)
        monkeypatch.setattr(M, name, f)
    ones = lambda t: torch.ones(t.shape, dtype=torch.float32)  # noqa: E731
    record("moara_token_logps", lambda x, lab, scale, entropy: (ones(lab), 2 * ones(lab) if entropy else None,
                                                              torch.zeros(lab.numel(), 4, dtype=torch.float32)))
    record("moara_token_logps_backward", lambda x, lab, stats, g, scale, entropy, grad_entropy: torch.ones_like(x) * g[..., None])

    def filled(loss, value, *rest):
        loss.fill_(value)
        return rest
    record("moara_preference_loss", lambda cfg, x, ref, offsets, mask, loss: filled(
        loss, 7.0, torch.tensor([7.0, 0.5, 0.1]), torch.zeros(4), torch.zeros(5)))
    record("moara_preference_loss_backward", lambda cfg, x, slope, g, offsets, mask: ones(x) * g)
    record("moara_policy_loss", lambda cfg, x, a, loss, **kw: filled(loss, 3.0, torch.arange(6.0) + 3, torch.zeros(5)))
    record("moara_policy_loss_backward", lambda cfg, x, a, w, g, entropy=None, **kw: (ones(x) * g, None if entropy is None else -ones(x) * g))
    record("moara_balance_loss", lambda cfg, x, i, loss, **kw: filled(
        loss, 5.0, torch.tensor([5.0, 1.0, 0.0]), torch.zeros(1, 3, dtype=torch.int64), torch.zeros(5)))
    record("moara_balance_loss_backward", lambda cfg, x, slope, g, **kw: torch.ones_like(x) * g)
    return seen


def test_logps_of_any_axes_and_gradients_of_one_output(calls):
    for lead in ((3,), (2, 3), (2, 2, 3), ()):
        x = torch.randn(*lead, 5, requires_grad=True)
        lab = torch.zeros(lead, dtype=torch.int32)
        logp = L.token_logps(x, lab, temperature=2.0)
        assert logp.shape == lead and calls[-1][2] == dict(scale=0.5, entropy=False) and calls[-1][1][1].dtype == torch.int64
        logp.sum().backward()
        assert x.grad.shape == x.shape and calls[-1][2]["grad_entropy"] is None
        logp, H = L.token_logps(x, lab, entropy=True)
        assert logp.shape == H.shape == lead
        torch.autograd.grad(H.sum(), x)
        assert calls[-1][2]["grad_entropy"] is not None and not calls[-1][1][3].any()
    with pytest.raises(ValueError):
        L.token_logps(x, torch.zeros(2, dtype=torch.int64))
    view = torch.randn(2, 4, 5)
    L.token_logps(view[:, :-1], torch.zeros(2, 3, dtype=torch.int64))
    assert calls[-1][1][0].data_ptr() == view.data_ptr()         # not copied


def test_a_gradient_of_the_entropies_alone_whatever_the_default_type(calls):
    """The log-probabilities' gradient is then made here: of float32, as the library takes it."""
    from paper_2609_15037_amd import losses as L
    x = torch.zeros(4, 7, requires_grad=True)
    torch.set_default_dtype(torch.bfloat16)
    try:
        L.token_logps(x, torch.zeros(4, dtype=torch.int64), entropy=True)[1].sum().backward()
    finally:
        torch.set_default_dtype(torch.float32)
    assert calls[-1][1][3].dtype == torch.float32 and not calls[-1][1][3].any()


def test_a_gradient_of_a_gradient_is_refused(calls):
    """Not given as if the first gradient did not depend on its inputs; the first one itself may be had in that way."""
    from paper_2609_15037_amd import losses as L
    x = torch.zeros(4, 7, requires_grad=True)
    loss, about = L.policy_loss(M.moara_policy_default_config(), L.token_logps(x, torch.zeros(4, dtype=torch.int64))[None],
                                torch.ones(1, 4))
    g, = torch.autograd.grad(loss, x, create_graph=True)
    assert torch.equal(g, torch.ones(4, 7))
    with pytest.raises(RuntimeError, match="no gradient of their gradient"):
        (loss + g.square().sum()).backward()


def test_losses_are_scalars_of_their_own(calls):
    """A loss changed in place leaves what it came with; gradients arrive scaled; a configuration changed between forward
    and backward stays what it was."""
    x = torch.randn(4, 3, requires_grad=True)
    cfg = M.moara_preference_config(beta=0.1)
    loss, rewards, about = L.preference_loss(cfg, x)
    cfg.beta = 9.0
    loss /= 4
    assert float(about[0]) == 7 and float(loss.detach()) == 1.75 and not about.requires_grad and not rewards.requires_grad
    loss.backward()
    assert calls[-1][1][0].beta == 0.1 and torch.equal(x.grad, torch.full_like(x, 0.25))
    cfg = M.moara_policy_config(clip_low=0.2)
    H = torch.randn(4, 3, requires_grad=True)
    loss, about = L.policy_loss(cfg, x, torch.ones(4, 3, dtype=torch.float64), entropy=H)
    assert calls[-1][1][2].dtype == torch.float32
    cfg.clip_low = 0.9
    gx, gh = torch.autograd.grad(loss, [x, H])
    assert calls[-1][1][0].clip_low == 0.2 and torch.equal(gx, torch.ones_like(x)) and torch.equal(gh, -torch.ones_like(x))
    loss, about = L.policy_loss(cfg, x, torch.ones(4, 3), entropy=H.detach())
    torch.autograd.grad(loss, x)
    assert calls[-1][2]["entropy"] is None              # no gradient that nobody takes
    loss, counts, about = L.balance_loss(M.moara_balance_config(experts=3, top_k=1), x, torch.zeros(4, 1, dtype=torch.int32))
    assert not counts.requires_grad
    (2 * loss).backward()
    with pytest.raises(RuntimeError):
        torch.autograd.grad(torch.autograd.grad(L.preference_loss(cfg, x)[0], x, create_graph=True)[0].sum(), x)


# ---------------------------------------------------------------- the performance cases

def _cases():
    import importlib.util
    import random
    from tests.conftest import ROOT
    spec = importlib.util.spec_from_file_location("more_operators", os.path.join(ROOT, "perf", "more_operators.py"))
    cases = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(cases)
    r = random.Random(5)
    return cases, cases.listed() + [cases.draw(r) for _ in range(300)]


def test_the_performance_cases_name_what_the_library_has(lib):
    """Every listed case and drawn ones get the configuration that they describe."""
    assert M.MOARA_KL_CUBIC == M.MOARA_KL_EXP
    cases, every = _cases()
    seen = set()
    for case in every:
        if case["op"] in ("logps",):
            continue
        cfg = cases._config(case)
        if case["op"] in ("policy", "policy_step"):
            kl = case.get("kl", "exp")
            seen.add(kl)
            assert cfg.kl == {"linear": M.MOARA_KL_LINEAR, "square": M.MOARA_KL_SQUARE}.get(kl, M.MOARA_KL_EXP)
            assert cfg.kl_coef == (0 if kl == "none" else case.get("kl_coef", 0.04))
        elif case["op"] == "preference":
            assert (cfg.beta, cfg.margin, cfg.smoothing, cfg.average) == (case["beta"], case["margin"], case["smoothing"], case["average"])
        else:
            assert (cfg.experts, cfg.top_k, cfg.z_coef) == (case["experts"], case["top_k"], case["z_coef"])
    assert len(seen) >= 4


# ---------------------------------------------------------------- alignment of vector accesses

@pytest.mark.parametrize("source", ["logps.hip", "loss.hip", "balance.hip", "route.hip", "adamw.hip"])
def test_vectors_are_accessed_with_the_alignment_they_are_declared_with(source):
    """Rows begin at any element. An access that the compiler takes for more aligned than its pointer's type is an error."""
    import subprocess
    from paper_2609_15037_amd import build
    try:
        hipcc = build.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    r = subprocess.run([hipcc, *build._flags(), "-Werror=align-mismatch", "--cuda-device-only", "-fsyntax-only",
                        os.path.join(build.CSRC, source)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]


# ---------------------------------------------------------------- workspace sizes

def test_workspaces_of_sizes_given_as_int(tmp_path):
    """The header's macros count in 64 bits whatever type a C program's sizes have, and as the binding does."""
    import shutil
    import subprocess
    from tests.conftest import ROOT
    gcc = shutil.which("gcc")
    if not gcc:
        pytest.skip("no C compiler")
    sizes = [(8, 0, 1), (64, 16384, 1), (256, 32768, 16), (1024, 1 << 24, 4), (64, 2 ** 31 - 1, 2), (1024, 2 ** 31 - 1, 1 << 21)]
    lines = "".join(f"  {{ int e = {e}, t = {t}, s = {s}; printf(\"%lld %lld\\n\", (long long)MOARA_BALANCE_WORKSPACE(e, t, s), "
                    f"(long long)MOARA_LOSS_WORKSPACE(t, s)); }}\n" for e, t, s in sizes)
    src = tmp_path / "sizes.c"
    src.write_text("#include <stdio.h>\n#include \"moara.h\"\nint main(void) {\n" + lines + "  return 0;\n}\n")
    subprocess.run([gcc, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "sizes")], check=True, capture_output=True)
    got = subprocess.run([str(tmp_path / "sizes")], check=True, capture_output=True, text=True).stdout.split()
    want = []
    for e, t, s in sizes:
        want += [(8 * e + 64) * (2 * s + t // 32 + 2), 0 if s + (t + 255) // 256 <= 17 else 48 * (s + t // 512 + 130)]
    assert [int(x) for x in got] == want


# ---------------------------------------------------------------- masks and offsets of a training program

def test_masks_and_offsets_of_other_types_and_layouts(calls):
    """A mask beside `logits[:, :-1]` is `mask[:, 1:]`, often of integers, and offsets may be int32: the losses take them as they
    take log-probabilities, forward and backward; ones that the library takes are passed on as they are."""
    whole = torch.tensor([[1, 1, 0, 1, 1], [1, 0, 0, 1, 2]] * 2)
    want = whole[:, 1:].ne(0)
    x = torch.randn(4, 4, requires_grad=True)
    pre, pol, adv = M.moara_preference_config(beta=0.1), M.moara_policy_config(), torch.ones(4, 4)
    bal, index = M.moara_balance_config(experts=4, top_k=1), torch.zeros(4, 1, dtype=torch.int32)

    def passed(call, key):
        call.backward()
        for _, a, kw in calls[-2:]:
            yield kw[key]
    for kind in (torch.int64, torch.int32, torch.uint8, torch.bool):
        mask = (whole != 0 if kind == torch.bool else whole).to(kind)[:, 1:]
        for loss in (L.preference_loss(pre, x, mask=mask)[0], L.policy_loss(pol, x, adv, mask=mask)[0]):
            for m in passed(loss, "mask"):
                assert m.is_contiguous() and m.dtype in (torch.bool, torch.uint8) and torch.equal(m != 0, want)
        for m in passed(L.balance_loss(bal, x, index, mask=mask[:, 1])[0], "mask"):
            assert m.is_contiguous() and m.dtype in (torch.bool, torch.uint8) and torch.equal(m != 0, want[:, 1])
    for same in (want.contiguous(), want.to(torch.uint8)):
        assert next(passed(L.preference_loss(pre, x, mask=same)[0], "mask")) is same
    flat = torch.randn(16, requires_grad=True)
    for o in (torch.tensor([0, 4, 16], dtype=torch.int32), torch.tensor([0, 1, 4, 1, 16])[::2]):
        for loss in (L.preference_loss(pre, flat, offsets=o)[0], L.policy_loss(pol, flat, flat.detach(), offsets=o)[0],
                     L.balance_loss(bal, x, index, offsets=o)[0]):
            for got in passed(loss, "offsets"):
                assert got.dtype == torch.int64 and got.is_contiguous() and torch.equal(got, o.long())
    o = torch.tensor([0, 16])
    assert next(passed(L.preference_loss(pre, flat, offsets=o)[0], "offsets")) is o
    for mask in (torch.ones(4, 4), torch.zeros(4, 4, dtype=torch.bfloat16)):       # 1 and 0, or 0 and -infinity: not guessed
        with pytest.raises(ValueError, match="mask"):
            L.preference_loss(pre, x, mask=mask)
