"""Plain forms of the worker-side operators in 64 bits (numpy), and bounds on what fp32 arithmetic may add.

The bounds count roundings, before any result was seen.  u = 2^-24 is half a step of fp32.  A term 2^((l - m) k) of a row
carries the rounding of the difference, of k (log2 e, 1 / temperature and their product) and of the product with k -- 5 u
of the exponent, in natural units 5 u |z - max z| -- and 2 u of the exponential itself; a sum of n terms in a chain adds n u.
log s turns the relative error of s into an absolute one; the difference with the taken logit, its scaling and the
logarithm's own rounding stay below 4 u of the numbers themselves.
"""
import numpy as np

U = 2.0 ** -24
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def counts(targets, vocab, weights=None):
    c = (targets >= 0) & (targets < vocab)
    return c if weights is None else c & (weights != 0)


def rows(logits, targets, temperature, weights=None):
    """(logp, lse, p, counts, bound on logp) of float64 logits."""
    T, V = logits.shape
    live = counts(targets, V, weights)
    logp, lse, p, bound = np.zeros(T), np.zeros(T), np.zeros((T, V)), np.zeros(T)
    for t in np.nonzero(live)[0]:
        z = logits[t] / temperature
        m = z.max()
        e = np.exp(z - m)
        s = e.sum()
        logp[t], lse[t], p[t] = z[targets[t]] - m - np.log(s), m + np.log(s), e / s
        seen = z[z > -1e30]
        # the exponent's error weighs with the term; chains of at most V / 64 + 64 terms (a wave a row, or more)
        spread = float((e / s * np.minimum(m - z, 1e30)).sum()) if len(seen) else 0.0
        far = m - z[targets[t]]
        bound[t] = U * (5 * spread + 2 + V / 64 + 64 + 4 * far + 4 * np.log(V) + 2 * abs(logp[t]) + 2 * abs(lse[t]))
    return logp, lse, p, live, bound


def policy_terms(logp, old, ref, adv, low, high, kl):
    r = np.exp(logp - old)
    held = np.clip(r, 1 - low, 1 + high)
    free, fixed = -adv * r, -adv * held
    clipped = free < fixed
    loss, slope = np.where(clipped, fixed, free), np.where(clipped, 0.0, free)
    k = np.zeros_like(loss)
    size = np.abs(np.where(clipped, 0.0, free))
    if kl:
        d = ref - logp
        k = np.expm1(d) - d
        loss, slope = loss + kl * k, slope - kl * np.expm1(d)
        size = size + kl * (np.exp(d) + np.abs(d))
    return loss, k, clipped, slope, size


def dlogits_of(p, targets, live, c):
    d = -c[:, None] * p
    d[np.nonzero(live)[0], targets[live]] += c[live]
    return d


def gradient_bound(d, p, targets, live, c, c_error, logp_bound, dtype):
    """Bound on dlogits: p's relative error is that of its own exponent and of the sum; c's own error on top; the
    last rounding is the type's."""
    with np.errstate(divide="ignore"):
        far = np.where(p > 0, -np.log(np.maximum(p, 1e-300)), 0.0)
    onehot = np.zeros_like(p)
    onehot[np.nonzero(live)[0], targets[live]] = 1.0
    rel = U * (10 * far + 8) + 2 * logp_bound[:, None]
    b = np.abs(c)[:, None] * (p * rel + 4 * U * onehot) + np.abs(c_error)[:, None] * (p + onehot)
    return b + HALF_STEP[dtype] * (np.abs(d) + b) + 1e-38


def preference(logp, ref, live, weights, offsets, beta, smooth, scale):
    w = np.ones_like(logp) if weights is None else weights.astype(np.float64)
    away = np.where(live, (logp - ref) * w, 0.0)
    pairs = (len(offsets) - 1) // 2
    margins, c, loss = np.zeros(pairs), np.zeros_like(logp), 0.0
    for b in range(pairs):
        a, m, e = offsets[2 * b:2 * b + 3]
        s = beta * (away[a:m].sum() - away[m:e].sum())
        margins[b] = s
        loss += (1 - smooth) * np.logaddexp(0, -s) + smooth * np.logaddexp(0, s)
        sig = 1 / (1 + np.exp(-s))
        c[a:m] = scale * beta * (sig - (1 - smooth))
        c[m:e] = -c[a:m][0] if m > a else -scale * beta * (sig - (1 - smooth))
    return scale * loss, margins, np.where(live, c * w, 0.0)


# ---------------------------------------------------------------- kept activations
def kept(x):
    """Values that the 8-bit form of x (float32 [T, K]) stands for, and the exponents [blocks, K]."""
    T, K = x.shape
    blocks = (T + 31) // 32
    out, exps = np.zeros((T, K)), np.zeros((blocks, K), np.int64)
    for b in range(blocks):
        v = x[32 * b:32 * b + 32].astype(np.float64)
        ok = np.isfinite(v)
        most = np.abs(np.where(ok, v, 0.0)).max(axis=0)
        e = np.full(K, -117)
        while np.any(most > 448 * 2.0 ** e):
            e = np.where(most > 448 * 2.0 ** e, e + 1, e)
        exps[b] = e
        s = 2.0 ** e
        q = np.clip(np.where(ok, v, 0.0), -240 * 2.0 ** 120, 240 * 2.0 ** 120) / s
        with np.errstate(divide="ignore"):
            step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(q), 1e-300))), -6) - 3)
        out[32 * b:32 * b + 32] = np.where(ok, np.round(q / step) * step * s, np.nan)
    return out, exps


def packed_bytes(x):
    """The packed form of x, byte by byte."""
    T, K = x.shape
    B, C = (T + 31) // 32, (K + 15) // 16 * 16
    values, exps = kept(x)
    q = np.zeros((B, C, 32), np.uint8)
    table = {}
    for code in range(256):
        s, e, m = code >> 7, (code >> 3) & 15, code & 7
        if (e, m) != (15, 7):
            v = (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) * (-1 if s else 1)
            table[(v, s)] = code
    for t in range(T):
        for k in range(K):
            v = values[t, k] / 2.0 ** exps[t // 32, k]
            q[t // 32, k, t % 32] = table[(v, int(np.signbit(x[t, k])))]
    scales = np.zeros((B, C), np.uint8)
    scales[:, :K] = exps + 127
    return np.concatenate([q.reshape(-1), scales.reshape(-1)])
