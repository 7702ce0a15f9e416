"""The loss against a teacher's top logits, and its gradient, in float64 (numpy), row by row from
the definition, with the magnitudes that bound float32 errors.

Error bounds, u = 2^-24.  A base-2 exponential of z = (y - m) a has an argument off by at most
4 u |z| (difference, factor, product, the factor's own rounding), hence a relative error of
(4 |z| + 2) u; |z| 2^z <= 0.54, so against the row's largest term (2^0 = 1, in the sum) each
term is off by at most 5 u absolutely and (4 |z| + 2) u relatively.  Sums add their terms in chains
of at most 64 per thread and 24 joins: 90 u relative.  So every q is within
    u (K + 4 |z|) q,   K = 100,
of the exact one, and p likewise with its own z.  float32 has no normal number below
TINY = 2^-126: a smaller exponential (the row's largest is 1) may come out as 0, an absolute error of
TINY, and so may its product with a coefficient.  Values stored in bfloat16 add 2^-8 of
themselves.  The loss adds logarithms: 4 u (|log| + K) for each of its terms."""
import numpy as np

U = 2.0 ** -24
K = 100
BF16 = 2.0 ** -8
TINY = 2.0 ** -126


def softmax(y):
    """(softmax, log softmax, |y - max| with infinities as 200) of one row; NaN as it comes."""
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        z = y - y.max()
        e = np.exp(z)
        s = e.sum()
        return e / s, z - np.log(s), np.minimum(np.abs(z), 200.0)


def distill(Y, ids, teacher, labels, T, soft_scale, hard_scale):
    """(G, loss[3], bound of G, bound of the loss[3]) of float64 operands."""
    n, C = Y.shape
    G, B = np.zeros((n, C)), np.zeros((n, C))
    soft = hard = esoft = ehard = 0.0
    for v in range(n):
        ok = (ids[v] >= 0) & (ids[v] < C) & ~(teacher[v] == -np.inf)
        if ok.any():
            q, lq, z = softmax(Y[v] / T)
            p, lp, zp = softmax(teacher[v][ok] / T)
            at = ids[v][ok]
            P, eP = np.zeros(C), np.zeros(C)
            np.add.at(P, at, p)
            np.add.at(eP, at, p * (K + 6 * zp))
            G[v] += soft_scale * T * (q - P)
            B[v] += abs(soft_scale) * T * U * (q * (K + 6 * z) + eP + 4 * np.abs(P)) + TINY * (1 + abs(soft_scale) * T)
            with np.errstate(invalid="ignore"):
                term = np.where(p > 0, p * (lp - lq[at]), 0.0 * p)
                soft += term.sum()
                size = np.where(p > 0, p * (np.abs(lp) + np.where(np.isfinite(lq[at]), np.abs(lq[at]), 0.0) + 1) * (K + 6 * zp), 0.0 * p)
                esoft += size.sum()
        if labels is not None and 0 <= labels[v] < C:
            q, lq, z = softmax(Y[v])
            G[v] += hard_scale * q
            G[v, labels[v]] -= hard_scale
            B[v] += abs(hard_scale) * U * q * (K + 6 * z) + TINY * (1 + abs(hard_scale))
            B[v, labels[v]] += 4 * U * abs(hard_scale)
            hard -= lq[labels[v]]
            ehard += K + 6 * (abs(lq[labels[v]]) if np.isfinite(lq[labels[v]]) else 0.0)
    soft, esoft = soft_scale * T * T * soft, abs(soft_scale) * T * T * esoft * U
    hard, ehard = hard_scale * hard, abs(hard_scale) * ehard * U
    loss = np.array([soft + hard, soft, hard])
    return G, loss, B, np.array([esoft + ehard, esoft, ehard]) + 2 * U * np.abs(loss)
