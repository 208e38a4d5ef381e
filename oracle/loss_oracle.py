"""Float64 oracle of the losses: log-probabilities of tokens, pairs of responses, a clipped policy, load balancing of
routing. NumPy, written from the definitions; shares no code with the library."""
from __future__ import annotations

import math

import numpy as np


# ---------------------------------------------------------------- log-probabilities of tokens

def log_softmax(x):
    with np.errstate(all="ignore"):
        a = x - x.max(axis=-1, keepdims=True)
        e = np.exp(a)
        # the largest, 1, apart from the others: the logarithm of 1 plus their sum is good also where that is tiny
        np.put_along_axis(e, np.argmax(x, axis=-1)[..., None], 0.0, axis=-1)
        bad = np.isnan(a).any(axis=-1, keepdims=True)
        return np.where(bad, np.nan, a - np.log1p(e.sum(axis=-1, keepdims=True)))


def xlogy(p, log):
    """p log, 0 where p is 0."""
    return np.where(p == 0, 0.0, p * np.where(p == 0, 0.0, log))


def token_logps(logits, labels, scale=1.0):
    """(log-probabilities, entropies); 0 for labels outside the vocabulary."""
    log = log_softmax(logits * scale)
    on = (labels >= 0) & (labels < logits.shape[-1])
    at = np.where(on, labels, 0)[..., None]
    logp = np.where(on, np.take_along_axis(log, at, -1)[..., 0], 0.0)
    return logp, np.where(on, -xlogy(np.exp(log), log).sum(axis=-1), 0.0)


def token_logps_grad(logits, labels, grad_logp, grad_entropy=None, scale=1.0):
    log = log_softmax(logits * scale)
    p = np.exp(log)
    on = (labels >= 0) & (labels < logits.shape[-1])
    g = np.where(on, grad_logp, 0.0)[..., None]
    hit = np.arange(logits.shape[-1]) == np.where(on, labels, -1)[..., None]
    out = g * np.where(hit, -np.expm1(log), -p)
    if grad_entropy is not None:
        H = -xlogy(p, log).sum(axis=-1, keepdims=True)
        out = out - np.where(on, grad_entropy, 0.0)[..., None] * xlogy(p, log + H)
    out = scale * out
    return np.where(on[..., None] & ((g != 0) | (0 if grad_entropy is None else np.asarray(grad_entropy)[..., None] != 0)), out, 0.0)


# ---------------------------------------------------------------- packed sequences

def members(tokens, sequences, offsets=None, mask=None):
    """Of each sequence the indices of its tokens that are not masked."""
    if offsets is None:
        offsets = np.arange(sequences + 1) * (tokens // sequences)
    on = np.ones(tokens, bool) if mask is None else np.asarray(mask).reshape(-1).astype(bool)
    out = []
    for a, b in zip(offsets[:-1], offsets[1:]):
        t = np.arange(a, b)
        out.append(t[on[a:b]])
    return out


# ---------------------------------------------------------------- pairs of responses

def log1p_exp(z):
    return np.logaddexp(0.0, z)


def preference_pair(h, kind, beta, margin=0.0, smoothing=0.0):
    """(loss, its derivative) of a pair's h."""
    z = beta * h - margin
    if kind == "sigmoid":
        return (1 - smoothing) * log1p_exp(-z) + smoothing * log1p_exp(z), beta * (smoothing - np.exp(-log1p_exp(z)))
    if kind == "hinge":
        return max(0.0, 1 - z), (-beta if z < 1 else 0.0)
    return (h - 1 / (2 * beta)) ** 2, 2 * (h - 1 / (2 * beta))


def preference(logp, ref, seqs, kind="sigmoid", beta=0.1, margin=0.0, smoothing=0.0, average=False):
    """(loss, share ahead, mean beta h), rewards, gradient of logp; all flat, seqs as members() gives them."""
    d = logp - (0.0 if ref is None else ref)
    D = np.array([math.fsum(d[t]) / (len(t) if average and len(t) else 1) for t in seqs])
    rows, grad, slopes = [], np.zeros_like(logp), []
    for p in range(len(seqs) // 2):
        a, b = seqs[2 * p], seqs[2 * p + 1]
        if not len(a) + len(b):
            continue
        h = D[2 * p] - D[2 * p + 1]
        l, dl = preference_pair(h, kind, beta, margin, smoothing)
        rows.append((l, float(h > 0), beta * h))
        slopes += [(a, dl), (b, -dl)]
    n = max(1, len(rows))
    for t, s in slopes:
        if len(t):
            grad[t] = s / n / (len(t) if average else 1)
    out = np.array(rows).reshape(-1, 3).sum(axis=0) / n
    return out, beta * D, grad


# ---------------------------------------------------------------- clipped policy

def policy_terms(logp, old, ref, adv, low, high, kl="exp"):
    """By token: gain, its slope, distance to the reference, its slope, clipped, distance to the old policy."""
    with np.errstate(all="ignore"):
        d = np.zeros_like(logp) if old is None else logp - old
        r = np.exp(d)
        clipped = ((r > 1 + high) & (adv > 0)) | ((r < 1 - low) & (adv < 0))
        none = (adv == 0) & ~np.isnan(r)        # no part, whatever the ratio
        gain = np.where(none, 0.0, np.where(clipped, np.where(adv > 0, 1 + high, 1 - low), r) * adv)
        slope = np.where(clipped | none, 0.0, r * adv)
        if ref is None:
            far = dfar = np.zeros_like(logp)
        else:
            q = ref - logp
            far, dfar = {"exp": lambda: (np.expm1(q) - q, -np.expm1(q)), "linear": lambda: (-q, np.ones_like(q)),
                         "square": lambda: (q * q / 2, -q)}[kl]()
        return gain, slope, far, dfar, clipped, np.expm1(d) - d


def policy_weights(seqs, reduce="tokens", divisor=0.0):
    """Weight of a sequence's tokens in the mean."""
    n = np.array([len(t) for t in seqs], float)
    over = divisor or (n.sum() if reduce == "tokens" else (n > 0).sum())
    w = np.where(n > 0, 1.0 if reduce == "tokens" else 1 / np.maximum(n, 1), 0.0)
    return w / over if over else w * 0


def policy(logp, old, ref, adv, entropy, seqs, low=0.2, high=0.2, kl="exp", kl_coef=0.0, entropy_coef=0.0, reduce="tokens",
           divisor=0.0):
    """out (6), weights, gradients of logp and of the entropies; flat; adv of each token."""
    gain, slope, far, dfar, clipped, moved = policy_terms(logp, old, ref, adv, low, high, kl)
    weight = policy_weights(seqs, reduce, divisor)
    w = np.zeros_like(logp)
    for t, x in zip(seqs, weight):
        w[t] = x
    on = w > 0
    mean = lambda x: math.fsum((w * np.where(on, x, 0.0))[on])  # noqa: E731
    policy_, kl_, ent = -mean(gain), mean(far), 0.0 if entropy is None else mean(entropy)
    times = lambda c, x: c * x if c else 0.0  # noqa: E731     a coefficient of 0 leaves its term out, whatever it is
    out = np.array([policy_ + times(kl_coef, kl_) - times(entropy_coef, ent), policy_, kl_, ent, mean(clipped), mean(moved)])
    return out, weight, np.where(on, w * (times(kl_coef, np.where(on, dfar, 0)) - np.where(on, slope, 0)), 0.0), \
        np.where(on, -entropy_coef * w, 0.0)


# ---------------------------------------------------------------- load balancing

def balance_scores(logits, sigmoid):
    """Scores (a sigmoid's over their sum) and which tokens have any."""
    with np.errstate(all="ignore"):
        if sigmoid:
            log = np.minimum(logits, 0) - np.log1p(np.exp(-np.abs(logits)))
            e = np.exp(log - log.max(axis=1, keepdims=True))
            s = e / e.sum(axis=1, keepdims=True)
        else:
            s = np.exp(log_softmax(logits))
    there = ~np.isnan(s).any(axis=1)
    return np.where(there[:, None], s, 0.0), there


def balance(logits, index, seqs, sigmoid=False, balance_coef=0.01, z_coef=0.0, load=None):
    """out (3), counts, gradient of the logits; seqs as members() gives them."""
    T, E = logits.shape
    s, there = balance_scores(logits, sigmoid)
    seqs = [t[there[t]] for t in seqs]
    counts = np.array([np.bincount(index[t][(index[t] >= 0) & (index[t] < E)].reshape(-1), minlength=E) for t in seqs],
                      dtype=np.int64).reshape(len(seqs), E)
    live = max(1, sum(len(t) > 0 for t in seqs))
    n = max(1, sum(len(t) for t in seqs))
    with np.errstate(all="ignore"):
        top = logits.max(axis=1)
        lse = top + np.log(np.exp(logits - top[:, None]).sum(axis=1))
        soft = np.exp(logits - lse[:, None])
    total, z, grad = 0.0, 0.0, np.zeros_like(logits)
    for t, c in zip(seqs, counts):
        if not len(t):
            continue
        c = c if load is None else np.asarray(load)
        f = E * c / c.sum() if c.sum() else np.zeros(E)
        total += float(f @ s[t].mean(axis=0)) / live
        if c.sum():         # a constant in f has no gradient, as scores sum to 1
            d = s[t] * ((f - 1) - (s[t] * (f - 1)).sum(axis=1, keepdims=True))
            if sigmoid:
                with np.errstate(all="ignore"):
                    d = d / (1 + np.exp(logits[t]))
            grad[t] += balance_coef * d / (len(t) * live)
        if z_coef:
            z += float((lse[t] ** 2).sum()) / n
            grad[t] += z_coef * 2 * lse[t][:, None] * soft[t] / n
    return np.array([balance_coef * total + z_coef * z, total, z]), counts, grad
