"""Plain forms in 64 bits (numpy) of what a worker that learns from a teacher calls -- alternatives with entropy, the distillation loss,
the root-mean-square norm -- and bounds on what the kernels' arithmetic may add.

The bounds count roundings, before any result was seen.  u = 2^-24 is half a step of fp32.  A term 2^((l - m) k) carries the rounding of the
difference, of k and of their product, 3 u of an exponent of size |z - max z| in natural units, and 2 u of the exponential; a chain of n
additions adds n u (a thread adds V / 256 terms at most, then come 8 additions over a wave and 16 over its workgroup: V / 64 + 64 holds all
of it)."""
import numpy as np

U = 2.0 ** -24
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def log_softmax(x64, temperature):
    z = x64 / temperature
    m = z.max()
    base = m if np.isfinite(m) else 0.0
    e = np.exp(z - base)
    return z - base - np.log(e.sum()), z, base


def sum_error(z, m, V):
    """Relative error of a sum of exp(z - m) over the words of z."""
    e = np.exp(z - m)
    s = e.sum()
    if s == 0.0:
        return 0.0
    gap = np.where(e > 0, m - z, 0.0)
    return U * (3 * float((e * gap).sum() / s) + 2 + V / 64 + 64)


def top(x64, k, temperature):
    """(ids, log-probabilities) of one row of float64 logits: the k largest finite ones, ties to the lower id."""
    order = np.argsort(-x64, kind="stable")
    order = order[x64[order] > -np.inf][:k]
    logp, _, _ = log_softmax(x64, temperature)
    ids, values = np.full(k, -1, np.int64), np.full(k, -np.inf)
    ids[:len(order)], values[:len(order)] = order, logp[order]
    return ids, values


def logp_error(x64, temperature):
    """Bound on a row's log-probabilities, word by word."""
    logp, z, m = log_softmax(x64, temperature)
    s = sum_error(z, m, len(x64))
    far = np.where(np.isfinite(z), m - z, 0.0)
    seen = np.where(np.isfinite(logp), np.abs(logp), 0.0)
    return s + U * (4 * far + 4 * np.log(len(x64)) + 2 * seen + 2)


def entropy(x64, temperature):
    """(H, bound).  H = log s + sum e (m - z) / s: the second sum's terms carry those of e (3 u (m - z) + 2 u) and 3 u of (m - z)
    itself and its product."""
    logp, z, m = log_softmax(x64, temperature)
    p = np.exp(logp)
    gap = np.where(p > 0, m - z, 0.0)
    H = float(-(p * np.where(p > 0, logp, 0.0)).sum())
    V = len(x64)
    second = float((p * gap).sum())
    own = U * float((p * gap * (3 * gap + 5 + V / 64 + 64)).sum())
    return H, own + sum_error(z, m, V) * (1 + second) + U * (4 * np.log(V) + 4 * second + 2)


def top_grad(x64, temperature, y, dlogp, dH, ids, dtop, dtype):
    """(gradient, bound) of one row; y, ids outside the row do not count."""
    V = len(x64)
    logp, z, m = log_softmax(x64, temperature)
    p = np.exp(logp)
    H, H_error = entropy(x64, temperature)
    D, sparse, size = dlogp, np.zeros(V), np.zeros(V)
    if dlogp:
        sparse[y] += dlogp
        size[y] += abs(dlogp)
    for i, d in zip(ids, dtop):
        if 0 <= i < V:
            D += d
            sparse[i] += d
            size[i] += abs(d)
    gap, lp = np.where(p > 0, m - z, 0.0), np.where(p > 0, logp, 0.0)
    want = (sparse - p * (D + dH * (lp + H))) / temperature
    rel = U * (3 * gap + 8) + sum_error(z, m, V)
    # lp + H = (z - m) - mean of it: each held to 4 u of its size and to the mean's own error
    inner = abs(dH) * (H_error + U * 6 * (gap + np.log(V) + H))
    bound = (p * rel * (abs(D) + abs(dH) * np.abs(lp + H)) + p * (inner + 4 * U * abs(D)) + 4 * U * size) / temperature
    return want, bound + HALF_STEP[dtype] * (np.abs(want) + bound) + 1e-38


class Distilled:
    """One token: kl, nll, gradient (unweighted) and bounds on them."""

    def __init__(self, x64, temperature, y, ids, tlogp, ce, renormalise):
        V = len(x64)
        logp, z, m = log_softmax(x64, temperature)
        p, q, named = np.exp(logp), np.zeros(V), np.zeros(V, bool)
        for i, t in zip(ids, np.asarray(tlogp, np.float64)):
            if 0 <= i < V and not named[i]:
                named[i], q[i] = True, np.exp(t)
        rest = p[~named].sum()
        share = q.sum()
        if renormalise:
            q, left = (q / share if share > 0 else q), 0.0
        else:
            left = max(0.0, 1.0 - share) if rest > 0 else 0.0
        Q = q.sum() + left
        on = q > 0
        with np.errstate(divide="ignore"):
            terms = q[on] * (np.log(q[on]) - logp[on])
            last = left * (np.log(left) - np.log(rest)) if left > 0 else 0.0
        self.kl = float(terms.sum() + last) if Q > 0 else 0.0
        self.nll = -logp[y] if y is not None else 0.0
        ratio = left / rest if rest > 0 else 0.0
        d = (Q + ce) * p - q
        d[~named] -= ratio * p[~named]
        if y is not None:
            d[y] -= ce
        self.d = d
        # the words named are formed in 64 bits from the sum over the others, whose relative error is e; one rounding to fp32 each
        zr = z[~named]
        mr = zr.max() if len(zr) and np.isfinite(zr.max()) else 0.0
        e = sum_error(zr, mr, V) if rest > 0 else 0.0
        gap = np.where(np.isfinite(z), np.abs(mr - z), 0.0)
        shift = e * rest
        b = np.where(named, (Q + ce) * p * (shift + U) + 2 * U * np.abs(d), p * ((Q + ce) + ratio) * (e + shift + U * (3 * gap + 6)))
        if y is not None:
            b[y] += 4 * U * ce
        self.d_error = b
        # f(d) = e^d - d - 1 is off by |p - q| times the error of d, and by 40 u of itself (its series, in fp32)
        with np.errstate(divide="ignore", invalid="ignore"):
            dist = np.where(on, np.abs(logp - np.log(np.where(on, q, 1.0))), 0.0)
            f = np.where(on, q * np.expm1(np.minimum(logp - np.log(np.where(on, q, 1.0)), 50.0)) - q * (logp - np.log(np.where(on, q, 1.0))),
                         np.where(named, p, 0.0))
        dist_r = abs(np.log(rest) - np.log(left)) if left > 0 and rest > 0 else 0.0
        f_r = rest - left - left * (np.log(rest) - np.log(left)) if left > 0 and rest > 0 else rest
        off = np.where(named, np.abs(p - q), 0.0)
        self.kl_error = float((off * (shift + U * dist)).sum() + abs(rest - left) * (e + shift + U * dist_r) +
                              40 * U * (np.abs(f).sum() + abs(f_r)) + 2 * U * abs(self.kl)) + 1e-15
        self.nll_error = e + U * (4 * abs(self.nll) + 4)


def norm(x, residual, gain, eps, to_type):
    """(h, y, rstd) in 64 bits, h rounded as it is stored."""
    h = x.astype(np.float64)
    if residual is not None:
        h = to_type((x.astype(np.float32) + residual.astype(np.float32)))
    rstd = 1.0 / np.sqrt((h * h).mean(axis=1) + eps)
    return h, h * rstd[:, None] * gain, rstd


def norm_grad(dy, h, gain, rstd, dres):
    """(dx, dgain, bound on dx but for its last rounding, sum of |dy h'|)."""
    K = h.shape[1]
    unit = h * rstd[:, None]
    a = dy * gain
    mean = (a * unit).sum(axis=1) / K
    dx = rstd[:, None] * (a - unit * mean[:, None])
    # dy g one rounding, h' two, the mean's terms 4 and its own rounding, then two products, a difference and a product
    size = np.abs(a * unit).sum(axis=1) / K
    bound = rstd[:, None] * U * (4 * np.abs(a) + np.abs(unit) * (8 * size[:, None] + 8 * np.abs(mean)[:, None]))
    if dres is not None:
        dx = dx + dres
        bound = bound + U * np.abs(dx)
    return dx, (dy * unit).sum(axis=0), bound, np.abs(dy * unit).sum(axis=0)
