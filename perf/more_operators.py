"""Performance cases of the losses whose gradients a training step takes.

Four operators of the library on the inputs a training program has, and one run of them together:

* ``logps``       : log-probabilities (and entropies) of given tokens under logits tokens x vocab, and the
                    gradient of the logits;
* ``preference``  : a loss of paired responses (chosen, rejected) over packed sequences, and its gradient;
* ``policy``      : the clipped policy loss with a penalty on the distance to a reference, and its gradient;
* ``balance``     : the load-balancing loss of expert routing with the experts' token counts, and its gradient;
* ``policy_step`` : from logits through ``logps`` and ``policy`` and back to the logits' gradient.

Every case is also computed in a plain form of elementary torch operations (``own`` false) and in 64 bits
(``exact``).

Definitions. With x = scale logits[t] and p = softmax(x): logp = log p[label], entropy = -sum p log p, both 0 for a
label outside the vocabulary. A pair's margin is h = D(chosen) - D(rejected) with D the sum (or mean) of logp - ref
over a sequence's tokens; its loss, of z = beta h - margin, (1 - smoothing) softplus(-z) + smoothing softplus(z), or
max(0, 1 - z), or (h - 1 / (2 beta))^2. A token's policy loss is -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A)
with r = exp(logp - old), and kl_coef times its distance to the reference, less entropy_coef times its entropy.
Balance: per sequence sum_e f_e P_e, f_e = E c_e / sum c of the tokens each expert was given and P_e the mean of its
scores; z: the mean of the squared log-sum-exp of a token's logits.
"""
import math

import torch

own = False

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
CLIP_LOW, CLIP_HIGH = 0.2, 0.28


# ---------------------------------------------------------------- cases

def _logps(name, tokens, vocab, dtype="bf16", entropy=False, train=True, scale=1.0, pad=0):
    """pad: columns behind the vocabulary in each row of logits."""
    return dict(name=name, op="logps", tokens=tokens, vocab=vocab, dtype=dtype, entropy=entropy, train=train, scale=scale,
                pad=pad)


def _preference(name, pairs, tokens, kind="sigmoid", average=False, smoothing=0.0, margin=0.0, beta=0.1, reference=True,
                mask=False, padded=False, tail=0):
    """tokens: of all sequences, which have lengths from 0 on; padded: sequences of equal length in rows, with a mask;
    tail: tokens behind the last sequence."""
    return dict(name=name, op="preference", pairs=pairs, tokens=tokens, kind=kind, average=average, smoothing=smoothing,
                margin=margin, beta=beta, reference=reference, mask=mask, padded=padded, tail=tail)


def _policy(name, sequences, tokens, reduce="tokens", per_sequence=True, kl="cubic", kl_coef=0.04, entropy_coef=0.0,
            old=True, mask=True, padded=False, tail=0):
    """kl: of the distance's estimators e^q - q - 1 (cubic), logp - ref (linear), its half square (square), or none."""
    return dict(name=name, op="policy", sequences=sequences, tokens=tokens, reduce=reduce, per_sequence=per_sequence, kl=kl,
                kl_coef=kl_coef, entropy_coef=entropy_coef, old=old, mask=mask, padded=padded, tail=tail)


def _balance(name, tokens, experts, top_k, score="softmax", dtype="f32", sequences=0, z_coef=0.0, mask=False):
    """sequences: packed ones, each balanced for itself; 0: all tokens together."""
    return dict(name=name, op="balance", tokens=tokens, experts=experts, top_k=top_k, score=score, dtype=dtype,
                sequences=sequences, z_coef=z_coef, mask=mask)


def _step(name, sequences, tokens, vocab, dtype="bf16"):
    return dict(name=name, op="policy_step", sequences=sequences, tokens=tokens, vocab=vocab, dtype=dtype)


def listed():
    return [
        # a few tokens scored under the 32000-word vocabulary of the Llama shapes, no gradient; latency
        _logps("logps_few", 8, 32000, train=False),
        # a reference model's log-probabilities of a batch: 8192 tokens, forward only
        _logps("logps_reference", 8192, 32000, train=False),
        # the trained model's: both directions, entropies for a bonus, fp32 logits, odd sizes and padded rows
        _logps("logps_ragged", 2039, 50021, "f32", entropy=True, scale=1.25, pad=27),
        # a large vocabulary, both directions: the largest call
        _logps("logps_large", 4096, 131072),
        # four pairs of short answers; latency
        _preference("preference_small", 4, 1000),
        # a large accumulated batch of packed pairs with masked prompts, length-normalised with a margin, no reference
        _preference("preference_packed", 1024, 2000000, average=True, margin=0.5, beta=2.0, reference=False, mask=True, tail=1000),
        # eight short answers in padded rows, advantages of whole answers; latency
        _policy("policy_small", 8, 8 * 100, padded=True),
        # a large rollout batch, packed; advantages of tokens, entropy bonus, sequences weighted alike
        _policy("policy_packed", 1024, 2000000, reduce="sequences", per_sequence=False, kl="square", entropy_coef=0.01, tail=1000),
        # the example's router: 8 experts, 512 tokens; latency
        _balance("balance_small", 512, 8, 2),
        # DeepSeek-MoE's router: 64 experts, top 6, padding tokens, both losses
        _balance("balance_64", 16384, 64, 6, z_coef=1e-3, mask=True),
        # a larger router of sigmoid scores, balanced within each of 16 packed sequences
        _balance("balance_256", 32768, 256, 8, score="sigmoid", sequences=16),
        # 32 answers from logits to the logits' gradient, as a training step runs it
        _step("policy_step_32000", 32, 4096, 32000),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    """One more case: 1 to 65536 tokens, vocabularies of 100 to 160000, 1 to 4096 sequences or pairs, 4 to 512 experts, up
    to the largest listed case's elements."""
    op = rng.choice(["logps", "logps", "logps", "preference", "preference", "policy", "policy", "balance", "balance",
                     "policy_step"])
    if op == "logps":
        vocab = _log(rng, 100, 160000)
        return _logps("", _log(rng, 1, min(65536, 250000000 // vocab)), vocab, rng.choice(["f32", "bf16"]), rng.random() < 0.4,
                      rng.random() < 0.7, rng.choice([1.0, 1.0, 1.25, 0.625]), rng.choice([0, 0, 0, 27, 64]))
    if op == "policy_step":
        vocab = _log(rng, 300, 131072)
        sequences = _log(rng, 1, 64)
        return _step("", sequences, max(sequences, _log(rng, 16, min(8192, 130000000 // vocab))), vocab, rng.choice(["f32", "bf16"]))
    if op == "balance":
        experts = _log(rng, 4, 512)
        tokens = _log(rng, 1, min(65536, 32768 * 256 // experts))
        return _balance("", tokens, experts, min(rng.randint(1, 12), experts - 1), rng.choice(["softmax", "sigmoid"]),
                        rng.choice(["f32", "bf16"]), rng.choice([0, 0, min(tokens, _log(rng, 1, 256))]), rng.choice([0.0, 1e-3]),
                        rng.random() < 0.4)
    count = _log(rng, 1, 2048)
    padded = rng.random() < 0.3
    tokens = _log(rng, 2 * count, 1000000)
    if op == "preference":
        if padded:
            tokens = tokens // (2 * count) * 2 * count
        kind = rng.choice(["sigmoid", "sigmoid", "hinge", "square"])
        return _preference("", count, tokens, kind, rng.random() < 0.4, rng.choice([0.0, 0.1]) if kind == "sigmoid" else 0.0,
                           rng.choice([0.0, 0.5]) if kind != "square" else 0.0, rng.choice([0.05, 0.1, 0.5]), rng.random() < 0.7,
                           padded or rng.random() < 0.5, padded, 0 if padded else rng.choice([0, 0, min(77, tokens // 4)]))
    if padded:
        tokens = tokens // count * count
    return _policy("", count, tokens, rng.choice(["tokens", "sequences"]), rng.random() < 0.6,
                   rng.choice(["cubic", "linear", "square", "none"]), rng.choice([0.001, 0.04, 0.2]), rng.choice([0.0, 0.01]),
                   rng.random() < 0.8, padded or rng.random() < 0.6, padded, 0 if padded else rng.choice([0, 0, min(77, tokens // 4)]))


# ---------------------------------------------------------------- inputs

class _State:
    pass


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * (seed + 1) + 7919)
    return gen


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _rand(gen, *shape):
    return torch.rand(*shape, generator=gen, device="cuda")


def _logits_and_labels(gen, tokens, vocab, dtype, pad=0):
    """Logits that spread over about e^6, the labels' among the larger ones; a tenth of the tokens has no label."""
    buf = torch.empty(tokens, vocab + pad, dtype=_DTYPE[dtype], device="cuda")
    buf.normal_(0.0, 2.0, generator=gen)
    labels = (_rand(gen, tokens) * vocab).long().clamp_(max=vocab - 1)
    buf.scatter_add_(1, labels[:, None], (_rand(gen, tokens, 1) * 14.0).to(buf.dtype))
    labels[_rand(gen, tokens) < 0.1] = -100
    return buf[:, :vocab], labels


def _offsets(gen, sequences, tokens, tail=0):
    """Bounds of packed sequences of any length from 0 on; `tail` more tokens follow the last."""
    cuts = (_rand(gen, sequences - 1) * (tokens - tail + 1)).long().sort()[0]
    ends = torch.tensor([0, tokens - tail], dtype=torch.int64, device="cuda")
    return torch.cat([ends[:1], cuts, ends[1:]])


def prepare(case, seed):
    st = _State()
    st.case = case
    gen = _generator(seed)
    op = case["op"]
    if op in ("logps", "policy_step"):
        st.logits, st.labels = _logits_and_labels(gen, case["tokens"], case["vocab"], case["dtype"], case.get("pad", 0))
    if op == "logps":
        T = case["tokens"]
        # gradients of a mean over the batch; clipped tokens have none
        st.grad_logp = _randn(gen, T).mul_(1.0 / T) * (_rand(gen, T) < 0.9)
        st.grad_entropy = torch.full((T,), -0.01 / T, device="cuda")
        return st
    if op == "balance":
        _prepare_balance(st, gen)
    elif op == "preference":
        _prepare_preference(st, gen)
    else:
        _prepare_policy(st, gen)
    if own:                 # the configuration a program makes once
        st.cfg = _config(case)
    return st


def _prepare_preference(st, gen):
    case = st.case
    T, S = case["tokens"], 2 * case["pairs"]
    st.logp = (1.0 - _rand(gen, T)).log_()
    st.ref = st.logp + 0.2 * _randn(gen, T) if case["reference"] else None
    st.mask = _rand(gen, T) < 0.7 if case["mask"] else None
    st.offsets = None if case["padded"] else _offsets(gen, S, T, case["tail"])
    if case["padded"]:
        st.logp, st.ref, st.mask = (None if x is None else x.view(S, T // S) for x in (st.logp, st.ref, st.mask))
    st.grad = torch.full((1,), 0.25, device="cuda")     # four accumulated batches


def _prepare_policy(st, gen):
    case = st.case
    T, S = case["tokens"], case["sequences"]
    st.logp = (1.0 - _rand(gen, T)).log_()
    if case["op"] == "policy_step":     # the logits of the rollout were nearly these
        exact = torch.log_softmax(st.logits.float(), dim=1).gather(1, st.labels.clamp(min=0)[:, None])[:, 0]
        st.logp = torch.where(st.labels >= 0, exact, 0.0)
    st.old = st.logp + 0.15 * _randn(gen, T) if case.get("old", True) else None
    st.ref = st.logp + 0.3 * _randn(gen, T) if case.get("kl") != "none" else None
    st.entropy = 3.0 * _rand(gen, T) if case.get("entropy_coef") else None
    st.mask = _rand(gen, T) < 0.7 if case.get("mask", True) else None
    if case["op"] == "policy_step":
        st.mask = st.labels >= 0
    st.advantages = _randn(gen, S if case.get("per_sequence", True) else T)
    st.offsets = None if case.get("padded") else _offsets(gen, S, T, case.get("tail", 0))
    if case.get("padded"):
        row = lambda x: None if x is None else x.view(S, T // S)  # noqa: E731
        st.logp, st.old, st.ref, st.entropy, st.mask = (row(x) for x in (st.logp, st.old, st.ref, st.entropy, st.mask))
        if not case["per_sequence"]:
            st.advantages = row(st.advantages)
    st.grad = torch.full((1,), 0.25, device="cuda")


def _prepare_balance(st, gen):
    case = st.case
    T, E, k = case["tokens"], case["experts"], case["top_k"]
    popular = _randn(gen, E)
    st.logits = _randn(gen, T, E).mul_(1.5).add_(popular).to(_DTYPE[case["dtype"]])
    st.mask = _rand(gen, T) < 0.95 if case["mask"] else None
    # the experts that routing with a little of a bias gave the tokens; none to those that are not routed
    st.index = (st.logits.float() + 0.1 * _randn(gen, E)).topk(k, dim=1)[1].to(torch.int32)
    if st.mask is not None:
        st.index = torch.where(st.mask[:, None], st.index, -1)
    st.offsets = _offsets(gen, case["sequences"], T) if case["sequences"] else None
    st.grad = torch.full((1,), 0.25, device="cuda")


def _config(case):
    from paper_2609_15037_amd import moara as M
    if case["op"] == "preference":
        kind = {"sigmoid": M.MOARA_PREF_SIGMOID, "hinge": M.MOARA_PREF_HINGE, "square": M.MOARA_PREF_SQUARE}[case["kind"]]
        return M.moara_preference_default_config(kind=kind, beta=case["beta"], margin=case["margin"], smoothing=case["smoothing"],
                                                 average=int(case["average"]))
    if case["op"] == "balance":
        score = M.MOARA_SIGMOID if case["score"] == "sigmoid" else M.MOARA_SOFTMAX
        return M.moara_balance_default_config(experts=case["experts"], top_k=case["top_k"], score=score, balance_coef=0.01,
                                              z_coef=case["z_coef"])
    kl = {"cubic": M.MOARA_KL_CUBIC, "linear": M.MOARA_KL_LINEAR, "square": M.MOARA_KL_SQUARE, "none": M.MOARA_KL_CUBIC}
    reduce = M.MOARA_MEAN_SEQUENCES if case.get("reduce") == "sequences" else M.MOARA_MEAN_TOKENS
    return M.moara_policy_default_config(clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl=kl[case.get("kl", "cubic")],
                                         kl_coef=0.0 if case.get("kl") == "none" else case.get("kl_coef", 0.04),
                                         entropy_coef=case.get("entropy_coef", 0.01), reduce=reduce,
                                         sequence_advantages=int(case.get("per_sequence", True)))


# ---------------------------------------------------------------- a pass

def run(st):
    op = st.case["op"]
    if own:
        return {"logps": _logps_own, "preference": _preference_own, "policy": _policy_own, "balance": _balance_own,
                "policy_step": _step_own}[op](st)
    return {"logps": _logps_plain, "preference": _preference_plain, "policy": _policy_plain, "balance": _balance_plain,
            "policy_step": _step_plain}[op](st)


def _logps_own(st):
    from paper_2609_15037_amd import moara as M
    case = st.case
    logp, entropy, stats = M.moara_token_logps(st.logits, st.labels, scale=case["scale"], entropy=case["entropy"])
    out = {"logp": logp, "entropy": entropy} if case["entropy"] else {"logp": logp}
    if case["train"]:
        out["grad"] = M.moara_token_logps_backward(st.logits, st.labels, stats, st.grad_logp, scale=case["scale"], entropy=entropy,
                                                   grad_entropy=st.grad_entropy if case["entropy"] else None)
    return out


def _preference_own(st):
    from paper_2609_15037_amd import moara as M
    out, rewards, slope = M.moara_preference_loss(st.cfg, st.logp, st.ref, offsets=st.offsets, mask=st.mask)
    grad = M.moara_preference_loss_backward(st.cfg, st.logp, slope, st.grad, offsets=st.offsets, mask=st.mask)
    return {"out": out, "rewards": rewards, "grad": grad}


def _policy_own(st):
    from paper_2609_15037_amd import moara as M
    out, weight = M.moara_policy_loss(st.cfg, st.logp, st.advantages, old_logp=st.old, ref_logp=st.ref, entropy=st.entropy,
                                      offsets=st.offsets, mask=st.mask)
    grad, grad_entropy = M.moara_policy_loss_backward(st.cfg, st.logp, st.advantages, weight, st.grad, old_logp=st.old,
                                                      ref_logp=st.ref, entropy=st.entropy, offsets=st.offsets, mask=st.mask)
    return {"out": out, "grad": grad} if grad_entropy is None else {"out": out, "grad": grad, "grad_entropy": grad_entropy}


def _balance_own(st):
    from paper_2609_15037_amd import moara as M
    out, counts, slope = M.moara_balance_loss(st.cfg, st.logits, st.index, offsets=st.offsets, mask=st.mask)
    grad = M.moara_balance_loss_backward(st.cfg, st.logits, slope, st.grad, offsets=st.offsets, mask=st.mask)
    return {"out": out, "counts": counts, "grad": grad}


def _step_own(st):
    from paper_2609_15037_amd import losses
    logits = st.logits.detach().requires_grad_()
    logp, entropy = losses.token_logps(logits, st.labels, entropy=True)
    loss, about = losses.policy_loss(st.cfg, logp, st.advantages, old_logp=st.old, ref_logp=st.ref, entropy=entropy,
                                     offsets=st.offsets, mask=st.mask)
    grad, = torch.autograd.grad(loss, logits)
    return {"logp": logp.detach(), "out": about, "grad": grad}


# ---------------------------------------------------------------- plain forms

def _logps_forward_plain(logits, labels, scale):
    """(x - max, its exponentials, their sum, which tokens have a label, the labels as indices, log-probabilities,
    entropies)."""
    x = logits.float() * scale
    x = x - x.amax(dim=1, keepdim=True)
    e = torch.exp(x)
    total = e.sum(dim=1, keepdim=True, dtype=torch.float64)     # where one token has nearly all, the others' sum matters
    there = (labels >= 0) & (labels < logits.shape[1])
    at = torch.where(there, labels, 0)[:, None]
    log = torch.log(total)
    logp = torch.where(there, (x.gather(1, at) - log)[:, 0], 0.0).float()
    entropy = (e * x).sum(dim=1, keepdim=True, dtype=torch.float64)
    entropy = torch.where(there, (log - entropy / total)[:, 0], 0.0).float()
    return x, e, total, there, at, logp, entropy


def _logps_backward_plain(forward, scale, grad_logp, grad_entropy, dtype):
    x, e, total, there, at, _, entropy = forward
    g = torch.where(there, grad_logp, 0.0)[:, None]
    p = e / total.float()
    grad = p * -g
    last = e.gather(1, at)
    last = g * ((total - last) / total).float()     # the label's: g (1 - p), also where p is nearly 1
    if grad_entropy is not None:
        h = torch.where(there, grad_entropy, 0.0)[:, None]
        bits = x - torch.log(total.float()) + entropy[:, None]
        grad = grad - h * p * bits
        last = last - h * (p * bits).gather(1, at)
    return (grad.scatter_(1, at, last) * scale).to(dtype)


def _logps_plain(st):
    case = st.case
    forward = _logps_forward_plain(st.logits, st.labels, case["scale"])
    out = {"logp": forward[5], "entropy": forward[6]} if case["entropy"] else {"logp": forward[5]}
    if case["train"]:
        out["grad"] = _logps_backward_plain(forward, case["scale"], st.grad_logp, st.grad_entropy if case["entropy"] else None,
                                            st.logits.dtype)
    return out


def _sequence_of(tokens, count, offsets, mask):
    """Each token's sequence, and which tokens are in one and not masked."""
    t = torch.arange(tokens, device="cuda")
    if offsets is None:
        seq, on = t // (tokens // count), torch.ones(tokens, dtype=torch.bool, device="cuda")
    else:
        seq = (torch.searchsorted(offsets, t, right=True) - 1).clamp(0, count - 1)
        on = (t >= offsets[0]) & (t < offsets[-1])
    return seq, on if mask is None else on & mask.view(-1)


def _sums(x, on, count, offsets):
    """Sums of the live tokens' values over each sequence, in 64 bits."""
    x = torch.where(on, x, 0.0).double()
    if offsets is None:
        return x.view(count, -1).sum(dim=1)
    upto = torch.cat([x.new_zeros(1), x.cumsum(dim=0)])
    return upto[offsets[1:]] - upto[offsets[:-1]]


def _row_sums(x, on, offsets):
    """Sums of the live tokens' rows over each sequence, in 64 bits: sequences x columns."""
    x = torch.where(on[:, None], x, 0.0).t().double()
    if offsets is None:
        return x.sum(dim=1)[None]
    upto = torch.cat([x.new_zeros(x.shape[0], 1), x.contiguous().cumsum(dim=1)], dim=1)
    return (upto[:, offsets[1:]] - upto[:, offsets[:-1]]).t()


def _softplus(z):
    return z.clamp(min=0.0) + torch.log1p(torch.exp(-z.abs()))


def _preference_plain(st):
    case = st.case
    T, P, beta, eps = case["tokens"], case["pairs"], case["beta"], case["smoothing"]
    seq, on = _sequence_of(T, 2 * P, st.offsets, st.mask)
    d = st.logp.reshape(-1).double()
    if st.ref is not None:
        d = d - st.ref.reshape(-1).double()
    count = _sums(on, on, 2 * P, st.offsets)
    per = 1.0 / count.clamp(min=1.0) if case["average"] else torch.ones_like(count)
    total = _sums(d, on, 2 * P, st.offsets) * per
    h = total[0::2] - total[1::2]
    z = beta * h - case["margin"]
    if case["kind"] == "sigmoid":
        loss = (1 - eps) * _softplus(-z) + eps * _softplus(z)
        dz = (eps - 1 + 1 / (1 + torch.exp(-z))) * beta
    elif case["kind"] == "hinge":
        loss = (1 - z).clamp(min=0.0)
        dz = torch.where(z < 1, -beta, 0.0)
    else:
        loss = (h - 0.5 / beta) ** 2
        dz = 2 * (h - 0.5 / beta)
    there = (count[0::2] + count[1::2]) > 0
    share = there.double() / there.sum().clamp(min=1)
    out = torch.stack([(loss * share).sum(), ((h > 0) * share).sum(), (beta * h * share).sum()])
    slope = torch.stack([dz * share, -dz * share], dim=1).view(-1) * per
    grad = torch.where(on, slope.float()[seq] * st.grad, 0.0)
    return {"out": out.float(), "rewards": (beta * total).float(), "grad": grad.view(st.logp.shape)}


def _low(q):
    """e^q - q - 1, in 64 bits (the terms cancel near 0)."""
    q = q.double()
    return torch.expm1(q) - q


def _policy_terms(case, logp, old, ref, entropy, advantages, seq, on, count, offsets, grad):
    """(loss and what it is made of, gradients of logp and of the entropies)."""
    coef = 0.0 if ref is None else case.get("kl_coef", 0.04)
    bonus = case.get("entropy_coef", 0.01)
    a = advantages[seq] if case.get("per_sequence", True) else advantages.reshape(-1)
    d = torch.zeros_like(logp, dtype=torch.float64) if old is None else logp.double() - old.double()
    high = (d > math.log1p(CLIP_HIGH)) & (a > 0)
    low = (d < math.log1p(-CLIP_LOW)) & (a < 0)
    ratio = torch.exp(d.float())
    gain = torch.where(high, (1 + CLIP_HIGH) * a, torch.where(low, (1 - CLIP_LOW) * a, ratio * a))
    slope = torch.where(high | low, 0.0, -ratio * a)
    if ref is None:
        far, dfar = torch.zeros_like(logp), torch.zeros_like(logp)
    else:
        q = ref.double() - logp.double()
        if case.get("kl", "cubic") == "cubic":
            far, dfar = _low(q), -torch.expm1(q)
        elif case["kl"] == "linear":
            far, dfar = -q, torch.ones_like(q)
        else:
            far, dfar = 0.5 * q * q, -q
    n = _sums(on, on, count, offsets)
    if case.get("reduce") == "sequences":
        weight = 1.0 / (n.clamp(min=1.0) * (n > 0).sum().clamp(min=1))
    else:
        weight = torch.ones_like(n) / n.sum().clamp(min=1.0)
    w = weight.float()[seq]
    mean = lambda x: (_sums(x, on, count, offsets) * weight).sum()  # noqa: E731
    bits = torch.zeros_like(logp) if entropy is None else entropy
    policy, kl, ent = -mean(gain), mean(far), mean(bits)
    out = torch.stack([policy + coef * kl - bonus * ent, policy, kl, ent, mean((high | low).double()), mean(_low(d))])
    grad_logp = torch.where(on, (slope + coef * dfar.float()) * w * grad, 0.0)
    grad_entropy = None if entropy is None else torch.where(on, -bonus * w * grad, 0.0)
    return out.float(), grad_logp, grad_entropy


def _policy_plain(st):
    case = st.case
    seq, on = _sequence_of(case["tokens"], case["sequences"], st.offsets, st.mask)
    old, ref, entropy = (None if x is None else x.reshape(-1) for x in (st.old, st.ref, st.entropy))
    out, grad, grad_entropy = _policy_terms(case, st.logp.reshape(-1), old, ref, entropy, st.advantages, seq, on,
                                            case["sequences"], st.offsets, st.grad)
    grad = grad.view(st.logp.shape)
    return {"out": out, "grad": grad} if grad_entropy is None else {"out": out, "grad": grad,
                                                                      "grad_entropy": grad_entropy.view(st.logp.shape)}


def _step_plain(st):
    case = st.case
    forward = _logps_forward_plain(st.logits, st.labels, 1.0)
    logp, entropy = forward[5], forward[6]
    seq, on = _sequence_of(case["tokens"], case["sequences"], st.offsets, st.mask)
    out, grad_logp, grad_entropy = _policy_terms(case, logp, st.old, st.ref, entropy, st.advantages, seq, on, case["sequences"],
                                                 st.offsets, 1.0)
    return {"logp": logp, "out": out, "grad": _logps_backward_plain(forward, 1.0, grad_logp, grad_entropy, st.logits.dtype)}


def _balance_plain(st):
    case = st.case
    T, E, S = case["tokens"], case["experts"], max(1, case["sequences"])
    seq, on = _sequence_of(T, S, st.offsets, st.mask)
    x = st.logits.float()
    top = x.amax(dim=1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(dim=1, keepdim=True)
    lse = torch.where(on, (top + torch.log(total))[:, 0], 0.0)
    if case["score"] == "sigmoid":
        s = 1 / (1 + torch.exp(-x))
        own_slope = s
        s = s / s.sum(dim=1, keepdim=True)
        own_slope = s * (1 - own_slope)
    else:
        s = own_slope = e / total
    there = (st.index >= 0) & on[:, None]
    given = torch.zeros_like(x).scatter_add_(1, st.index.clamp(min=0).long(), there.float())
    counts = _row_sums(given, on, st.offsets).long()
    n = _sums(on, on, S, st.offsets)
    score = _row_sums(s, on, st.offsets)
    f = E * counts.double() / counts.sum(dim=1, keepdim=True).clamp(min=1)
    each = (f * score).sum(dim=1) / n.clamp(min=1)
    sequences = (n > 0).sum().clamp(min=1)
    tokens = n.sum().clamp(min=1)
    balance = each.sum() / sequences
    z = (lse.double() ** 2).sum() / tokens
    out = torch.stack([0.01 * balance + case["z_coef"] * z, balance, z if case["z_coef"] else 0.0 * z])
    # scores sum to 1, so a constant in f has no gradient: without its mean nothing cancels where the load is nearly even
    slope = (0.01 * (f - f.mean(dim=1, keepdim=True)) / (n.clamp(min=1) * sequences)[:, None]).float()[seq]
    grad = own_slope * (slope - (slope * s).sum(dim=1, keepdim=True))
    if case["z_coef"]:
        grad = grad + (2 * case["z_coef"] / tokens).float() * lse[:, None] * (e / total)
    grad = torch.where(on[:, None], grad * st.grad, 0.0)
    return {"out": out.float(), "counts": counts, "grad": grad.to(st.logits.dtype)}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    """Each input read once, each output written once."""
    op, T = case["op"], case["tokens"]
    if op in ("logps", "policy_step"):
        n, train = T * case["vocab"], case.get("train", True)
        b = n * _SIZE[case["dtype"]] * (2 if train else 1) + 12 * T
        if op == "policy_step":
            return {"bytes": b + 9 * T, "flops": 12 * n}
        return {"bytes": b + 4 * T * (train + case["entropy"] * (1 + train)), "flops": n * (12 if train else 5)}
    if op == "balance":
        E = case["experts"]
        b = T * (2 * E * _SIZE[case["dtype"]] + 4 * case["top_k"] + case["mask"]) + max(1, case["sequences"]) * E * 8
        return {"bytes": b, "flops": 14 * T * E}
    if op == "preference":
        return {"bytes": T * (8 + 4 * case["reference"] + case["mask"]) + 8 * case["pairs"], "flops": 4 * T}
    each = 8 + case["mask"] + 4 * case["old"] + 4 * (case["kl"] != "none") + 8 * (case["entropy_coef"] > 0)
    return {"bytes": T * each + 4 * (case["sequences"] if case["per_sequence"] else T), "flops": 30 * T}


# ---------------------------------------------------------------- in 64 bits, from the definitions

def exact(case, seed):
    global own
    before, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = before
    return {"logps": _exact_logps, "preference": _exact_preference, "policy": _exact_policy, "balance": _exact_balance,
            "policy_step": _exact_step}[case["op"]](st)


def _exact_rows(logits, labels, scale, each):
    """each(rows, log-probabilities and entropies of those rows as functions of x, x) over a few rows at a time."""
    for a in range(0, logits.shape[0], 256):
        rows = slice(a, min(a + 256, logits.shape[0]))
        x = logits[rows].double().requires_grad_()
        log = torch.log_softmax(x * scale, dim=1)
        lab = labels[rows]
        live = (lab >= 0) & (lab < logits.shape[1])
        logp = log.gather(1, lab.masked_fill(~live, 0)[:, None]).squeeze(1).masked_fill(~live, 0.0)
        entropy = -(log.exp() * log).sum(dim=1).masked_fill(~live, 0.0)
        each(rows, logp, entropy, x)


def _exact_logps(st):
    case = st.case
    T, V = st.logits.shape
    logp, entropy = torch.zeros(2, T, dtype=torch.float64, device="cuda")
    grad = torch.zeros(T, V, dtype=torch.float64, device="cuda") if case["train"] else None

    def each(rows, lp, h, x):
        logp[rows], entropy[rows] = lp.detach(), h.detach()
        if grad is not None:
            value = (lp * st.grad_logp[rows].double()).sum()
            if case["entropy"]:
                value = value + (h * st.grad_entropy[rows].double()).sum()
            grad[rows], = torch.autograd.grad(value, x)
    _exact_rows(st.logits, st.labels, case["scale"], each)
    out = {"logp": logp, "entropy": entropy} if case["entropy"] else {"logp": logp}
    return out if grad is None else {**out, "grad": grad}


def _members(case, st, count):
    """A count x tokens one-hot of the sequences' live tokens as (sequence of each token, live)."""
    T = case["tokens"]
    if st.offsets is None:
        seq = torch.arange(count, device="cuda").repeat_interleave(T // count)
        live = torch.ones(T, dtype=torch.bool, device="cuda")
    else:
        seq = torch.arange(count, device="cuda").repeat_interleave(st.offsets.diff())
        live = torch.arange(T, device="cuda") < seq.numel()
        seq = torch.cat([seq, seq.new_zeros(T - seq.numel())])
    return seq, live if st.mask is None else live & st.mask.flatten()


def _total(x, seq, live, count):
    return torch.zeros(count, dtype=torch.float64, device="cuda").scatter_add(0, seq, x * live)


def _exact_preference(st):
    case = st.case
    S = 2 * case["pairs"]
    seq, live = _members(case, st, S)
    logp = st.logp.flatten().double().requires_grad_()
    d = logp if st.ref is None else logp - st.ref.flatten().double()
    n = _total(torch.ones_like(d), seq, live, S)
    D = _total(d, seq, live, S)
    if case["average"]:
        D = D / n.clamp(min=1)
    h = D.view(-1, 2)[:, 0] - D.view(-1, 2)[:, 1]
    z = case["beta"] * h - case["margin"]
    if case["kind"] == "sigmoid":
        loss = -(1 - case["smoothing"]) * torch.nn.functional.logsigmoid(z) - case["smoothing"] * torch.nn.functional.logsigmoid(-z)
    elif case["kind"] == "hinge":
        loss = torch.relu(1 - z)
    else:
        loss = (h - 1 / (2 * case["beta"])).square()
    live_pair = n.view(-1, 2).sum(dim=1) > 0
    mean = lambda x: x.double()[live_pair].sum() / max(1, int(live_pair.sum()))  # noqa: E731
    out = torch.stack([mean(loss), mean(h > 0), mean(case["beta"] * h)])
    grad, = torch.autograd.grad(out[0], logp)
    return {"out": out.detach(), "rewards": (case["beta"] * D).detach(), "grad": (grad * st.grad.double()).view(st.logp.shape)}


def _exact_policy_loss(case, st, logp, entropy, seq, live, count):
    a = st.advantages.double()[seq] if case.get("per_sequence", True) else st.advantages.flatten().double()
    d = logp - (logp.detach() if st.old is None else st.old.flatten().double())
    r = d.exp()
    gain = torch.minimum(r * a, r.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * a)
    clipped = ((r > 1 + CLIP_HIGH) & (a > 0)) | ((r < 1 - CLIP_LOW) & (a < 0))
    far = torch.zeros_like(d)
    if st.ref is not None:
        q = st.ref.flatten().double() - logp
        kind = case.get("kl", "cubic")
        far = q.expm1() - q if kind == "cubic" else -q if kind == "linear" else q.square() / 2
    n = _total(torch.ones_like(d), seq, live, count)
    if case.get("reduce") == "sequences":
        w = 1 / n.clamp(min=1)[seq] / max(1, int((n > 0).sum()))
    else:
        w = torch.full_like(d, 1 / max(1, int(n.sum())))
    mean = lambda x: (x.double() * w * live).sum()  # noqa: E731
    policy, kl, ent = -mean(gain), mean(far), mean(entropy)
    coef = case.get("kl_coef", 0.04) if st.ref is not None else 0.0
    loss = policy + coef * kl - case.get("entropy_coef", 0.01) * ent
    return loss, torch.stack([loss, policy, kl, ent, mean(clipped), mean(d.expm1() - d)]).detach()


def _exact_policy(st):
    case = st.case
    seq, live = _members(case, st, case["sequences"])
    logp = st.logp.flatten().double().requires_grad_()
    entropy = torch.zeros_like(logp) if st.entropy is None else st.entropy.flatten().double()
    entropy = entropy.detach().requires_grad_()
    loss, out = _exact_policy_loss(case, st, logp, entropy, seq, live, case["sequences"])
    grad, grad_entropy = (g * st.grad.double() for g in torch.autograd.grad(loss, [logp, entropy]))
    found = {"out": out, "grad": grad.view(st.logp.shape)}
    return found if st.entropy is None else {**found, "grad_entropy": grad_entropy.view(st.logp.shape)}


def _exact_step(st):
    case = st.case
    T, V = st.logits.shape
    logp, entropy = torch.zeros(2, T, dtype=torch.float64, device="cuda")

    def forward(rows, lp, h, x):
        logp[rows], entropy[rows] = lp.detach(), h.detach()
    _exact_rows(st.logits, st.labels, 1.0, forward)
    logp.requires_grad_(), entropy.requires_grad_()
    seq, live = _members(case, st, case["sequences"])
    loss, out = _exact_policy_loss(case, st, logp, entropy, seq, live, case["sequences"])
    grads = torch.autograd.grad(loss, [logp, entropy])
    grad = torch.zeros(T, V, dtype=torch.float64, device="cuda")

    def backward(rows, lp, h, x):
        grad[rows], = torch.autograd.grad((lp * grads[0][rows]).sum() + (h * grads[1][rows]).sum(), x)
    _exact_rows(st.logits, st.labels, 1.0, backward)
    return {"logp": logp.detach(), "out": out, "grad": grad}


def _exact_balance(st):
    case = st.case
    E, S = case["experts"], max(1, case["sequences"])
    seq, live = _members(case, st, S)
    x = st.logits.double().requires_grad_()
    s = torch.softmax(x, dim=1)
    if case["score"] == "sigmoid":
        s = torch.sigmoid(x) / torch.sigmoid(x).sum(dim=1, keepdim=True)
    n = _total(torch.ones(case["tokens"], dtype=torch.float64, device="cuda"), seq, live, S)
    mean = torch.zeros(S, E, dtype=torch.float64, device="cuda").index_add(0, seq, s * live[:, None]) / n.clamp(min=1)[:, None]
    given = torch.nn.functional.one_hot(seq, S).double().T @ \
        (torch.nn.functional.one_hot((st.index + 1).long(), E + 1).sum(dim=1)[:, 1:].double() * live[:, None])
    f = E * given / given.sum(dim=1, keepdim=True).clamp(min=1)
    balance = (f * mean).sum() / max(1, int((n > 0).sum()))
    z = (torch.logsumexp(x, dim=1).square() * live).sum() / max(1, int(n.sum())) if case["z_coef"] else 0.0 * balance
    loss = 0.01 * balance + case["z_coef"] * z
    grad, = torch.autograd.grad(loss, x)
    return {"out": torch.stack([loss, balance, z]).detach(), "counts": None, "grad": grad * st.grad.double()}
