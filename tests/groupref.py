"""Group norms with an activation over the graphs of a batch in float64 (numpy), with the magnitudes that bound
float32 errors.

Error bounds.  u = 2^-24.  The statistics are float64 and add nothing that counts.  A normed element is
((x - hi) - lo) r: two differences of relative error u each (the second takes off what is below the first's last
place), r rounded once, a product; the weight's product and the bias's sum add u each, so that p is off by at most
6 u |u w| + u (|u w| + |b|) <= K u M with M = |u w| + |b| and K = 8.  ReLU adds nothing.  SiLU's slope is at most 1.1,
and its own arithmetic (exp within 2 ulp, a sum, a division) adds 5 u |y|.

Backward, d = dY act'(p): act' of SiLU is at most 1.1 and its own slope at most 1/2, so that d is off by at most
K u M / 2 |dY| + 10 u |dY|; a ReLU decides by float64 and is exact.  With Md = |dY| (2 + M / 2) for SiLU (|dY| else) every
further stage is linear: t = w d, the two means, the difference and the product with r; KB = 32 of u times the magnitudes'
own expression covers their at most ten roundings and the errors above.  A value stored in bfloat16 is off by another 2^-8."""
import numpy as np

U = 2.0 ** -24
K, KB = 8, 32
BF16 = 2.0 ** -8


def segments(ptr, n):
    return [(0, n)] if ptr is None else list(zip(ptr[:-1], ptr[1:]))


def statistics(X, ptr, G, eps):
    n, F = X.shape
    out = []
    for lo, hi in segments(ptr, n):
        x = X[lo:hi].reshape(hi - lo, G, F // G)
        if hi > lo:
            m = x.mean((0, 2))
            v = ((x - m[None, :, None]) ** 2).mean((0, 2))
        else:
            m = v = np.zeros(G)
        out.append(np.stack([m, 1.0 / np.sqrt(v + eps)], 1))
    return np.array(out)


def act(p, kind):
    if kind == "relu":
        return np.where(p > 0, p, 0.0)
    if kind == "silu":
        return p / (1.0 + np.exp(-p))
    return p


def slope(p, kind):
    if kind == "relu":
        return (p > 0).astype(float)
    if kind == "silu":
        q = 1.0 / (1.0 + np.exp(-p))
        return q + p * q * (1.0 - q)
    return np.ones_like(p)


def _vectors(w, b, F):
    return (np.ones(F) if w is None else w), (np.zeros(F) if b is None else b)


def forward(X, ptr, G, w, b, kind, eps):
    """(Y, bound, stats, rows): rows marks those of graphs."""
    n, F = X.shape
    w, b = _vectors(w, b, F)
    st = statistics(X, ptr, G, eps)
    Y, E, rows = np.zeros((n, F)), np.zeros((n, F)), np.zeros(n, bool)
    for (lo, hi), s in zip(segments(ptr, n), st):
        s = np.repeat(s, F // G, 0)
        p = (X[lo:hi] - s[:, 0]) * s[:, 1] * w + b
        Y[lo:hi] = act(p, kind)
        E[lo:hi] = 1.1 * K * U * (np.abs(p - b) + np.abs(b)) + 5 * U * np.abs(Y[lo:hi])
        rows[lo:hi] = True
    return Y, E, st, rows


def backward(X, dY, ptr, G, w, b, kind, eps):
    """((dX, bound), (dw, bound), (db, bound), rows)."""
    n, F = X.shape
    w, b = _vectors(w, b, F)
    st = statistics(X, ptr, G, eps)
    dX, E, rows = np.zeros((n, F)), np.zeros((n, F)), np.zeros(n, bool)
    dw, db, Mw, Mb = (np.zeros(F) for _ in range(4))
    for (lo, hi), s in zip(segments(ptr, n), st):
        if hi <= lo:
            continue
        r = np.repeat(s[:, 1], F // G)
        u = (X[lo:hi] - np.repeat(s[:, 0], F // G)) * r
        p = u * w + b
        d = dY[lo:hi] * slope(p, kind)
        Md = np.abs(dY[lo:hi]) * (2.0 + 0.5 * (np.abs(u * w) + np.abs(b)) if kind == "silu" else 1.0)
        mean = lambda a: np.repeat(a.reshape(hi - lo, G, F // G).mean((0, 2)), F // G)  # noqa: E731
        t, Mt = w * d, np.abs(w) * Md
        dX[lo:hi] = r * (t - mean(t) - u * mean(t * u))
        E[lo:hi] = r * (Mt + mean(Mt) + np.abs(u) * mean(Mt * np.abs(u)))
        dw, Mw = dw + (d * u).sum(0), Mw + (Md * np.abs(u)).sum(0)
        db, Mb = db + d.sum(0), Mb + Md.sum(0)
        rows[lo:hi] = True
    return (dX, KB * U * E), (dw, KB * U * Mw), (db, KB * U * Mb), rows
