"""Performance cases of the operators a training step needs beside the projected matrices' update.

Four operators of the library on the inputs a training program has:

* ``norm``  : the norm of all gradients and the coefficient that clips them to ``max_norm``;
* ``clip``  : the same, and the gradients scaled in place;
* ``adamw`` : one AdamW step over many tensors (embedding, output head, norms, expert routers), its
              moments in 32 bits, or in 8 bits with a scale for each 32 elements;
* ``route`` : routing of tokens to experts, its backward pass, the experts' token counts and the
              step of the balancing bias.

Parameters, gradients and moments are views of flat buffers, as sharded optimizers keep them; a
pass returns these buffers. Every case is also computed in a plain form of elementary torch
operations (``own`` false) and in 64 bits (``exact``).

8-bit moments, as both forms read and write them. A tensor's elements are cut into blocks of 32. With
e the biased binary exponent of the block's largest finite magnitude, one more where its significand is
over 1.75, and at least 18 (first moment) or 35 (second):

* first moment: E4M3 codes to nearest, of the value over 2^(e - 135);
* second moment: unsigned E5M3 codes, value (8 + f) 2^(E - 1) (f where E = 0) times 2^(e - 160) for the
  code 8 E + f, rounded up with the probability that makes its mean exact, the last 16 bits of a
  probability being random(i) of the element's index i; never to 0 where the value is not 0; 254 is
  the largest, 255 stands for NaN;
* a first moment that is not finite has the code 0x7f.

Two bytes for each block hold e of the first moment and of the second.
"""
import math

import torch

own = False

BETA1, BETA2, EPS, LR, MAX_NORM = 0.9, 0.999, 1e-6, 1e-4, 1.0
STEP = 1000
BLOCK = 32
_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------- cases

def _grads(name, op, layers, d, ffn, kv, experts, dtype, shift=0):
    """Gradients of `layers` layers of q, o (d x d), k, v (kv x d) and gate, up, down of `experts` MLPs
    of width ffn; with `shift` the tensors start at elements that are no multiple of anything."""
    return dict(name=name, op=op, layers=layers, d=d, ffn=ffn, kv=kv, experts=experts, dtype=dtype, shift=shift)


def _adamw(name, vocab, d, layers, bits, param, grad, routed=0, decay=0.0, clip=False, shift=0):
    """Embedding and head (vocab x d), 2 layers + 1 norms (d), `layers` router weights (routed x d)."""
    return dict(name=name, op="adamw", vocab=vocab, d=d, layers=layers, bits=bits, param=param, grad=grad,
                routed=routed, decay=decay, clip=clip, shift=shift)


def _route(name, tokens, experts, top_k, groups=1, top_groups=1, group_best=1, score="softmax", renorm=False,
           scale=1.0, bias=False, mask=False, dtype="f32", train=True):
    return dict(name=name, op="route", tokens=tokens, experts=experts, top_k=top_k, groups=groups,
                top_groups=top_groups, group_best=group_best, score=score, renorm=renorm, scale=scale, bias=bias,
                mask=mask, dtype=dtype, train=train)


def listed():
    return [
        # gradients of the smallest model of the repository's workloads: one fp32 layer of d = 256; latency
        _grads("norm_tiny_f32", "norm", 1, 256, 688, 256, 1, "f32"),
        # Llama-2-7B shapes, bf16 gradients, four layers (the norm is linear in them)
        _grads("norm_llama2_7b", "norm", 4, 4096, 11008, 4096, 1, "bf16"),
        # DeepSeek-MoE shapes: 202 matrices of one layer's experts, clipped before the projected update
        _grads("clip_deepseek_moe", "clip", 1, 2048, 1408, 2048, 66, "f32"),
        # sizes that are no multiple of anything, tensors that start anywhere in a flat buffer
        _grads("clip_ragged", "clip", 6, 1000, 2666, 500, 1, "bf16", shift=1),
        # the small Llama of the training-loop tests: five norms, embedding and head of 512 x 256; latency
        _adamw("adamw32_tiny_f32", 512, 256, 2, 32, "f32", "f32"),
        # the 300M stack's other parameters, a bf16 model with the clipping coefficient applied on the way
        _adamw("adamw32_llama_300m", 32000, 1024, 24, 32, "bf16", "bf16", clip=True),
        # the same, moments in 8 bits
        _adamw("adamw8_llama_300m", 32000, 1024, 24, 8, "bf16", "bf16", clip=True),
        # Llama-2-7B's: 2 x 131 M elements, the largest call
        _adamw("adamw8_llama2_7b", 32000, 4096, 32, 8, "bf16", "bf16"),
        # fp32 master weights with bf16 gradients, routers of 64 experts, decay, ragged sizes, odd starts
        _adamw("adamw8_ragged", 32003, 1000, 28, 8, "f32", "bf16", routed=64, decay=0.1, shift=1),
        # a few sequences decoding one token each, DeepSeek-MoE's 6 of 64; latency
        _route("route_decode", 8, 64, 6, dtype="bf16", train=False),
        # a training batch of DeepSeek-MoE's router: softmax scores, no renormalisation, padding tokens
        _route("route_train_64", 16384, 64, 6, mask=True),
        # a larger batch on 256 experts in 8 groups: sigmoid scores, balancing bias, renormalised weights
        _route("route_train_256", 32768, 256, 8, groups=8, top_groups=4, group_best=2, score="sigmoid", renorm=True,
               scale=2.5, bias=True),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    """One more case: widths 64 to 4096, vocabularies 300 to 64000, 1 to 65536 tokens, 8 to 512 experts,
    every type, up to the largest listed cases' element counts."""
    op = rng.choice(["norm", "clip", "adamw", "adamw", "adamw", "route", "route", "route"])
    if op in ("norm", "clip"):
        d = _log(rng, 64, 4096)
        d -= d % rng.choice([1, 2, 8, 64])
        ffn = int(d * rng.uniform(1.0, 4.5))
        kv = max(16, d // rng.choice([1, 4, 8]))
        experts = rng.choice([1, 1, 1, 8, 66])
        per = 2 * d * d + 2 * kv * d + 3 * experts * ffn * d
        most = 8.0e8 if op == "norm" else 5.5e8
        if per > most:
            experts, per = 1, 2 * d * d + 2 * kv * d + 3 * ffn * d
        layers = max(1, min(32, int(math.exp(rng.uniform(0.0, math.log(max(1.5, most / per)))))))
        return _grads("", op, layers, d, ffn, kv, experts, rng.choice(["f32", "bf16"]), rng.choice([0, 0, 1]))
    if op == "adamw":
        d = _log(rng, 64, 4096)
        d -= d % rng.choice([1, 2, 8, 64])
        vocab = _log(rng, 300, 64000)
        vocab = min(vocab, int(1.3e8 / d))
        param = rng.choice(["f32", "bf16"])
        return _adamw("", vocab, d, rng.randint(1, 32), rng.choice([8, 32]), param,
                      rng.choice(["bf16", "f32"]), routed=rng.choice([0, 0, 8, 64]), decay=rng.choice([0.0, 0.1]),
                      clip=rng.random() < 0.5, shift=rng.choice([0, 0, 1]))
    experts = _log(rng, 8, 512)
    groups = rng.choice([1, 1, 2, 4, 8])
    experts = max(groups * 2, experts - experts % groups)
    top_groups = rng.randint(1, groups)
    top_k = min(rng.randint(1, 12), experts // groups * top_groups)
    tokens = _log(rng, 1, min(65536, 32768 * 256 // experts))
    return _route("", tokens, experts, top_k, groups, top_groups, rng.choice([1, 2]), rng.choice(["softmax", "sigmoid"]),
                  rng.random() < 0.5, rng.choice([1.0, 2.5]), rng.random() < 0.5, rng.random() < 0.3,
                  rng.choice(["f32", "bf16"]), rng.random() < 0.7)


# ---------------------------------------------------------------- inputs

class _State:
    pass


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * (seed + 1) + 4241)
    return gen


def _flat(shapes, dtype, shift):
    """One zero buffer and the views of the shapes in it: starts on 128 elements, or just anywhere."""
    starts, end = [], shift
    for s in shapes:
        starts.append(end)
        n = math.prod(s)
        end += n + 7 - n % 2 if shift else -(-n // 128) * 128
    buf = torch.zeros(end, dtype=dtype, device="cuda")
    return buf, [buf[a:a + math.prod(s)].view(s) for a, s in zip(starts, shapes)]


def _grad_shapes(case):
    d, f, kv = case["d"], case["ffn"], case["kv"]
    one = [(d, d), (kv, d), (kv, d), (d, d)] + [(f, d), (f, d), (d, f)] * case["experts"]
    return one * case["layers"]


def _adamw_shapes(case):
    d = case["d"]
    out = [(case["vocab"], d)]
    for _ in range(case["layers"]):
        out += [(d,), (d,)] + ([(case["routed"], d)] if case["routed"] else [])
    return out + [(d,), (case["vocab"], d)]


def _seed64(case, seed):
    return (seed * 2654435761 + 97) % (1 << 63)


def prepare(case, seed):
    st = _State()
    st.case, st.seed = case, seed
    gen = _generator(seed)
    if case["op"] == "route":
        return _prepare_route(st, gen)
    if case["op"] == "adamw":
        return _prepare_adamw(st, gen)
    st.flat, st.grads = _flat(_grad_shapes(case), _DTYPE[case["dtype"]], case["shift"])
    for g in st.grads:      # rows of different sizes, norms well above the limit
        rows = torch.randn(g.shape[0], 1, generator=gen, device="cuda").exp_()
        g.copy_(torch.randn(g.shape, generator=gen, device="cuda").mul_(rows).mul_(1e-2))
    if own:                 # the marshalled pointers a training loop keeps while its gradients stay in place
        from paper_2609_15037_amd import moara as M
        st.args = M.GradArgs(st.grads)
    return st


def _prepare_adamw(st, gen):
    case = st.case
    shapes = _adamw_shapes(case)
    st.p, st.params = _flat(shapes, _DTYPE[case["param"]], case["shift"])
    g, st.grads = _flat(shapes, _DTYPE[case["grad"]], case["shift"])
    mdt = torch.float32 if case["bits"] == 32 else torch.uint8
    st.m, st.exp_avgs = _flat(shapes, mdt, case["shift"])
    st.v, st.exp_avg_sqs = _flat(shapes, mdt, case["shift"])
    counts = [2 * -(-math.prod(s) // BLOCK) for s in shapes]
    st.s = torch.zeros(sum(counts), dtype=torch.uint8, device="cuda")
    st.scales = list(st.s.split(counts))
    st.clip = torch.full((1,), 0.37, dtype=torch.float32, device="cuda") if case["clip"] else None
    st.decay = [case["decay"] if len(s) > 1 else 0.0 for s in shapes]
    for i, (p, g, m, v) in enumerate(zip(st.params, st.grads, st.exp_avgs, st.exp_avg_sqs)):
        p.copy_(torch.randn(p.shape, generator=gen, device="cuda").mul_(0.02) if p.dim() > 1 else torch.ones_like(p))
        # rows (tokens) of different frequency; an embedding has no gradient for tokens that did not occur
        rows = torch.randn(p.shape[0], generator=gen, device="cuda").exp_().mul_(1e-3)
        seen = torch.rand(p.shape[0], generator=gen, device="cuda") < (0.3 if i == 0 else 1.1)
        wide = [-1] + [1] * (p.dim() - 1)
        g.copy_(torch.randn(p.shape, generator=gen, device="cuda").mul_((rows * seen).view(wide)))
        m32 = torch.randn(p.shape, generator=gen, device="cuda").mul_(0.2 * rows.view(wide))
        v32 = torch.rand(p.shape, generator=gen, device="cuda").add_(0.5).mul_(rows.square().view(wide))
        if case["bits"] == 32:
            m.copy_(m32), v.copy_(v32)
        else:
            mc, vc, sc = _encode(m32.view(-1), v32.view(-1), _random16(p.numel(), 0, i))
            m.view(-1).copy_(mc), v.view(-1).copy_(vc), st.scales[i].copy_(sc)
    if own:                 # the marshalled pointers an optimizer keeps while its tensors stay in place
        from paper_2609_15037_amd import moara as M
        st.args = M.AdamWArgs(st.params, st.grads, st.exp_avgs, st.exp_avg_sqs, st.scales if case["bits"] == 8 else None,
                              weight_decay=st.decay)
        st.cfg = M.moara_adamw_config(beta1=BETA1, beta2=BETA2, eps=EPS, bits=case["bits"])
    return st


def _prepare_route(st, gen):
    case = st.case
    T, E = case["tokens"], case["experts"]
    popular = torch.randn(E, generator=gen, device="cuda")
    st.logits = torch.randn(T, E, generator=gen, device="cuda").mul_(1.5).add_(popular).to(_DTYPE[case["dtype"]])
    st.bias = torch.randn(E, generator=gen, device="cuda").mul_(0.02) if case["bias"] else None
    st.mask = torch.rand(T, generator=gen, device="cuda") < 0.95 if case["mask"] else None
    st.counts = torch.zeros(E, dtype=torch.int64, device="cuda")
    st.grad_weight = torch.randn(T, case["top_k"], generator=gen, device="cuda")
    if own:
        from paper_2609_15037_amd import moara as M
        st.cfg = M.moara_route_config(experts=E, top_k=case["top_k"], groups=case["groups"],
                                      top_groups=case["top_groups"], group_best=case["group_best"],
                                      score=M.MOARA_SIGMOID if case["score"] == "sigmoid" else M.MOARA_SOFTMAX,
                                      renormalise=int(case["renorm"]), scale=case["scale"])
    return st


# ---------------------------------------------------------------- a pass

def run(st):
    op = st.case["op"]
    if op == "route":
        return _route_own(st) if own else _route_plain(st)
    if op == "adamw":
        (_adamw_own if own else _adamw_plain)(st)
        if st.case["bits"] == 32:
            return {"param": st.p, "exp_avg": st.m, "exp_avg_sq": st.v}
        # E4M3 codes are a torch type; the unsigned E5M3 codes and the exponents have none: whole numbers
        return {"param": st.p, "exp_avg": st.m.view(torch.float8_e4m3fn), "exp_avg_sq": st.v, "scales": st.s}
    norm = _norm_own(st) if own else _norm_plain(st)
    return {"norm": norm, "grads": st.flat} if op == "clip" else {"norm": norm}


def _norm_own(st):
    from paper_2609_15037_amd import moara as M
    norm = M.moara_grad_norm(None, MAX_NORM, args=st.args)      # (norm, coefficient)
    if st.case["op"] == "clip":
        M.moara_grad_scale(None, norm[1:], args=st.args)
    return norm


def _adamw_own(st):
    from paper_2609_15037_amd import moara as M
    M.moara_adamw_step(st.args, st.cfg, LR, STEP, clip=st.clip, seed=_seed64(st.case, st.seed))


def _route_own(st):
    from paper_2609_15037_amd import moara as M
    index, weight = M.moara_route(st.cfg, st.logits, bias=st.bias, mask=st.mask, counts=st.counts)
    if not st.case["train"]:
        return {"index": index, "weight": weight}
    grad = M.moara_route_backward(st.cfg, st.logits, index, st.grad_weight)
    if st.bias is not None:
        M.moara_route_balance(st.counts, st.bias, 1e-3)
    return {"index": index, "weight": weight, "grad": grad, "counts": st.counts, "bias": st.bias}


# ---------------------------------------------------------------- plain forms

def _norm_plain(st):
    norm = torch.stack([g.float().square().sum() for g in st.grads]).sum().sqrt()
    coef = (MAX_NORM / (norm + 1e-6)).clamp(max=1.0)
    coef = torch.where(torch.isfinite(norm), coef, float("nan"))
    if st.case["op"] == "clip":
        for g in st.grads:
            g.copy_(torch.where(torch.isnan(coef), 0.0, g.float() * coef))
    return torch.stack([norm, coef])


_A, _B, _C = 0x9E3779B1, 0x6A09E667, 0xB7E15163     # odd; digits of the golden ratio, sqrt 2 and e


def _mix(x):
    """Mixes 32 bits: of a number or of an int64 tensor that holds 32 bits."""
    x = ((x ^ (x >> 16)) * _A) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * _B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random16(n, seed, tensor):
    """16 random bits for each of a tensor's n elements: halves of 32 that two neighbours share."""
    k0 = _mix((seed & 0xFFFFFFFF) ^ _mix((seed >> 32) ^ _mix(tensor)))
    k1 = _mix(k0 ^ _C)
    x = torch.arange((n + 1) // 2, device="cuda")
    x = (x + (x >> 32) * _C + k0) & 0xFFFFFFFF
    x = (((x ^ (x >> 16)) * _A) & 0xFFFFFFFF) ^ k1
    x = ((x ^ (x >> 15)) * _B) & 0xFFFFFFFF
    x = x ^ (x >> 16)
    return torch.stack([x & 0xFFFF, x >> 16], dim=1).view(-1)[:n]


def _pow2(e):
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _blocks(x):
    pad = -x.numel() % BLOCK
    return (torch.cat([x, x.new_zeros(pad)]) if pad else x).view(-1, BLOCK)


def _decode(mc, vc, scales):
    """The two moments, fp32, of a tensor's codes."""
    n = mc.numel()
    e = scales.view(-1, 2).to(torch.int32)
    m = _blocks(mc).view(torch.float8_e4m3fn).float() * _pow2(e[:, :1] - 135)
    c = _blocks(vc).to(torch.int32)
    base = torch.where(c >= 8, (8 + (c & 7)) * _pow2((c >> 3) - 1), c.float())
    v = torch.where(c == 255, float("nan"), base * _pow2(e[:, 1:] - 160))
    return m.view(-1)[:n], v.view(-1)[:n]


def _exponent(x, least):
    top = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(dim=1, keepdim=True)
    return ((top.view(torch.int32) + 0x1FFFFF) >> 23).clamp(least, 254)


def _encode(m, v, random16):
    n = m.numel()
    m, v, r = _blocks(m), _blocks(v), _blocks(random16.to(torch.int32)) << 4
    em, ev = _exponent(m, 18), _exponent(v, 35)
    mc = (m * _pow2(135 - em)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
    mc = torch.where(torch.isfinite(m), mc, 0x7F)
    w = v * _pow2(160 - ev)         # the value in units of the lowest code
    low = ((w * 1048576.0).clamp(max=8388608.0).round().to(torch.int32) + r) >> 20
    c = torch.where(w < 8, low, ((w.view(torch.int32) + r) >> 20) - 1032)
    c = torch.maximum(c, (v > 0).to(torch.int32)).clamp(max=254)
    c = torch.where(torch.isfinite(v), c, 255)
    scales = torch.cat([em, ev], dim=1).to(torch.uint8)
    return mc.view(-1)[:n], c.to(torch.uint8).view(-1)[:n], scales.view(-1)


def _adamw_plain(st):
    bits = st.case["bits"]
    b1, b2 = 1 - BETA1 ** STEP, 1 - BETA2 ** STEP
    for i, (p, g, m, v) in enumerate(zip(st.params, st.grads, st.exp_avgs, st.exp_avg_sqs)):
        g = g.float().view(-1)
        if st.clip is not None:
            g = g * st.clip
        m32, v32 = (m.view(-1), v.view(-1)) if bits == 32 else _decode(m.view(-1), v.view(-1), st.scales[i])
        m32 = m32 * BETA1 + g * (1 - BETA1)
        v32 = v32 * BETA2 + (g * g) * (1 - BETA2)
        step = (m32 / b1) / ((v32 / b2).sqrt() + EPS)
        p.copy_((p.float().view(-1) * (1 - LR * st.decay[i]) - LR * step).view(p.shape))
        if bits == 8:
            m32, v32, scales = _encode(m32, v32, _random16(p.numel(), _seed64(st.case, st.seed), i))
            st.scales[i].copy_(scales)
        m.view(-1).copy_(m32), v.view(-1).copy_(v32)


def _best(c, k):
    """Values and indices of the k largest of each row, the lowest index first among equals."""
    value, index = torch.sort(c, dim=-1, descending=True, stable=True)
    return value[..., :k], index[..., :k]


def _scores(case, logits):
    if case["score"] == "sigmoid":
        return 1 / (1 + torch.exp(-logits))
    e = torch.exp(logits - logits.amax(dim=-1, keepdim=True))
    # summed in 64 bits: the order of a sum must not decide between experts that are nearly equal
    return e / e.sum(dim=-1, keepdim=True, dtype=torch.float64).float()


def _route_plain(st):
    case = st.case
    T, E, k, G = case["tokens"], case["experts"], case["top_k"], case["groups"]
    none = float("-inf")
    logits = st.logits.float()
    s = _scores(case, logits)
    c = s if st.bias is None else s + st.bias
    c = torch.where(torch.isnan(c), none, c)
    if st.mask is not None:
        c = torch.where(st.mask[:, None], c, none)
    if G > 1:
        in_group, _ = _best(c.view(T, G, E // G), min(case["group_best"], E // G))
        group = torch.where(in_group == none, 0.0, in_group).sum(dim=-1)
        group = torch.where(in_group[..., 0] == none, none, group)
        _, kept = _best(group, case["top_groups"])
        on = torch.zeros(T, G, dtype=torch.bool, device="cuda").scatter_(1, kept, True)
        c = torch.where(on[:, :, None], c.view(T, G, E // G), none).view(T, E)
    value, index = _best(c, k)
    there = value != none
    weight = _weights(case, logits, s, index, there) * case["scale"]
    chosen = torch.where(there, index, -1).to(torch.int32)
    if not case["train"]:
        return {"index": chosen, "weight": weight}
    st.counts.scatter_add_(0, index.reshape(-1), there.reshape(-1).long())
    grad = _route_grad_plain(case, logits, s, index, there, weight / case["scale"], st.grad_weight)
    if st.bias is not None:
        st.bias.add_(1e-3 * torch.sign(st.counts.sum() - st.counts * E).float())
        st.counts.zero_()
    return {"index": chosen, "weight": weight, "grad": grad.to(st.logits.dtype), "counts": st.counts, "bias": st.bias}


def _weights(case, logits, s, index, there):
    """Weights of the chosen experts, before the factor on all of them."""
    if not case["renorm"]:
        return torch.where(there, s.gather(1, index), 0.0)
    if case["score"] == "softmax":      # the softmax over the chosen logits
        at = torch.where(there, logits.gather(1, index), float("-inf"))
        u = torch.exp(at - at.amax(dim=1, keepdim=True))
    else:
        u = s.gather(1, index)
    u = torch.where(there, u, 0.0)
    total = u.sum(dim=1, keepdim=True)
    return torch.where(total > 0, u / total, 0.0)


def _route_grad_plain(case, logits, s, index, there, u, dw):
    dw = torch.where(there, dw, 0.0)
    rest = 1 / (1 + torch.exp(logits.gather(1, index))) if case["score"] == "sigmoid" else 1.0
    if case["renorm"]:
        t = u * (dw - (dw * u).sum(dim=1, keepdim=True)) * rest
    else:
        t = u * dw * rest
    t = torch.where(there, t * case["scale"], 0.0)
    grad = torch.zeros_like(logits).scatter_add_(1, index, t)
    if case["score"] == "softmax" and not case["renorm"]:
        grad = grad - torch.where(there.any(dim=1, keepdim=True), s * t.sum(dim=1, keepdim=True), 0.0)
    return grad


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    """Each input read once, each output written once."""
    if case["op"] == "route":
        T, E, k = case["tokens"], case["experts"], case["top_k"]
        size = 2 if case["dtype"] == "bf16" else 4
        b = T * (E * size + k * 8 + case["mask"]) + 4 * E * case["bias"]
        f = T * E * 6
        if case["train"]:
            b += T * (E * size + k * 4) + 16 * E + 4 * E * case["bias"]
            f += T * E * 2
        return {"bytes": b, "flops": f}
    shapes = _grad_shapes(case) if case["op"] in ("norm", "clip") else _adamw_shapes(case)
    n = sum(math.prod(s) for s in shapes)
    if case["op"] == "adamw":
        size = {"f32": 4, "bf16": 2}
        each = 2 * size[case["param"]] + size[case["grad"]] + (16 if case["bits"] == 32 else 4 + 4 / BLOCK)
        return {"bytes": int(n * each), "flops": 14 * n}
    size = 2 if case["dtype"] == "bf16" else 4
    return {"bytes": n * size * (2 if case["op"] == "clip" else 1), "flops": 2 * n if case["op"] == "norm" else 3 * n}


# ---------------------------------------------------------------- in 64 bits, from the definitions

def exact(case, seed):
    return {"route": _exact_route, "adamw": _exact_adamw}.get(case["op"], _exact_norm)(case, seed)


def _without_own(case, seed):
    """The case's inputs (the library's handles are not wanted here)."""
    global own
    before, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = before


def _exact_norm(case, seed):
    st = _without_own(case, seed)
    total = 0.0
    for g in st.grads:
        total += float((g.double() ** 2).sum())
    norm = math.sqrt(total)
    coef = min(1.0, MAX_NORM / (norm + 1e-6))
    pair = torch.tensor([norm, coef], dtype=torch.float64)
    return {"norm": pair, "grads": st.flat.double() * coef} if case["op"] == "clip" else {"norm": pair}


def _two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_e4m3(x):
    """x (64 bits, at most 448) to the nearest E4M3 value, ties to the even one."""
    _, e = torch.frexp(x)
    unit = _two_to((e - 4).clamp(min=-9))
    return (x / unit).round() * unit


def _exact_scale(x):
    frac, e = torch.frexp(x.abs().amax(dim=1, keepdim=True))         # x = frac 2^e, frac in [1/2, 1)
    return e + 126 + (frac > 0.875).int()


def _exact_adamw(case, seed):
    st = _without_own(case, seed)
    shapes = _adamw_shapes(case)
    out = {"param": torch.zeros(st.p.shape, dtype=torch.float64, device="cuda")}
    out["exp_avg"] = torch.zeros_like(out["param"])
    out["exp_avg_sq"] = torch.zeros_like(out["param"]) if case["bits"] == 32 else None
    clip = 1.0 if st.clip is None else float(st.clip)
    end = case["shift"]
    for i, s in enumerate(shapes):
        n = math.prod(s)
        at = slice(end, end + n)
        end += n + 7 - n % 2 if case["shift"] else -(-n // 128) * 128
        g = st.grads[i].reshape(-1).double() * clip
        if case["bits"] == 32:
            m, v = st.m[at].double(), st.v[at].double()
        else:
            e = st.scales[i].view(-1, 2).int().repeat_interleave(BLOCK, dim=0)[:n]
            m = st.m[at].view(torch.float8_e4m3fn).double() * _two_to(e[:, 0] - 135)
            c = st.v[at].int()
            high = c // 8
            v = (c % 8 + 8 * (high > 0)) * _two_to((high - 1).clamp(min=0) + e[:, 1] - 160)
        m = BETA1 * m + (1 - BETA1) * g
        v = BETA2 * v + (1 - BETA2) * g ** 2
        hat = (m / (1 - BETA1 ** STEP)) / ((v / (1 - BETA2 ** STEP)) ** 0.5 + EPS)
        p = st.params[i].reshape(-1).double()
        out["param"][at] = p - LR * st.decay[i] * p - LR * hat
        if case["bits"] == 32:
            out["exp_avg"][at], out["exp_avg_sq"][at] = m, v
        else:
            b = _blocks(m)
            e = _exact_scale(b).clamp(18, 254)
            out["exp_avg"][at] = _exact_e4m3(b * _two_to(135 - e)).view(-1)[:n]
    if case["bits"] == 8:
        out["scales"] = None
    return out


def _exact_route(case, seed):
    st = _without_own(case, seed)
    T, E, k, G = case["tokens"], case["experts"], case["top_k"], case["groups"]
    x = st.logits.double()
    s = torch.sigmoid(x) if case["score"] == "sigmoid" else torch.softmax(x, dim=1)
    c = s.clone() if st.bias is None else s + st.bias.double()
    if G > 1:
        c = c.view(T, G, E // G)
        score = c.topk(min(case["group_best"], E // G), dim=2)[0].sum(dim=2)
        off = torch.ones(T, G, 1, dtype=torch.bool, device="cuda")
        off.scatter_(1, score.topk(case["top_groups"], dim=1)[1][:, :, None], False)
        c = c.masked_fill(off, -9.0).view(T, E)
    index = c.topk(k, dim=1)[1]
    at = s.gather(1, index)
    total = at.sum(dim=1, keepdim=True) if case["renorm"] else torch.ones(T, 1, dtype=torch.float64, device="cuda")
    live = torch.ones(T, 1, device="cuda") if st.mask is None else st.mask[:, None]
    weight = case["scale"] * at / total * live
    if not case["train"]:
        return {"index": None, "weight": weight}
    dw = st.grad_weight.double() * live * case["scale"]
    # d weight / d s, then the scores' own derivative
    ds = dw / total
    if case["renorm"]:
        ds = ds - (dw * at).sum(dim=1, keepdim=True) / total ** 2
    full = torch.zeros_like(s).scatter_(1, index, ds)
    grad = full * s * (1 - s) if case["score"] == "sigmoid" else s * (full - (full * s).sum(dim=1, keepdim=True))
    out = {"index": None, "weight": weight, "grad": grad, "counts": None, "bias": None}
    if st.bias is not None:
        n = torch.bincount(index[live[:, 0] > 0].reshape(-1), minlength=E).double()
        out["bias"] = st.bias.double() + 1e-3 * torch.sign(n.mean() - n)
    return out
