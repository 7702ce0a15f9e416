"""The norms around a block in float64 (numpy), with the magnitudes that bound float32 errors.

Error bounds.  u = 2^-24.  A sum over a row's F elements is formed in chains of at most 8
additions inside a thread, 6 between lanes and 15 between wavefronts, so its relative error is at
most 30 u of the sum of magnitudes; the reciprocal root adds 1 ulp, each product, sum and
conversion u.  A normed element's error is therefore at most K u times
    M = rho (|x| + mean|x|)          (>= |unit|)
with K = 64, and every further stage is linear in the magnitudes below.  The backward pass
nests two such stages (the stream's gradient, then the block's): K_BACK = 128.  A value stored in
bfloat16 is off by another 2^-8 of itself (half a step)."""
import numpy as np

U = 2.0 ** -24
K, K_BACK = 64, 128
BF16 = 2.0 ** -8


def unit(x, layer, eps):
    c = x - x.mean(1, keepdims=True) if layer else x
    rho = 1.0 / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    return c * rho, rho, rho * (np.abs(x) + (np.abs(x).mean(1, keepdims=True) if layer else 0.0))


def one(w, F):
    return np.ones(F) if w is None else w


def zero(b, F):
    return np.zeros(F) if b is None else b


def gate_values(gate, sigmoid, shape):
    if gate is None:
        return np.ones(shape)
    g = np.broadcast_to(gate, shape)
    return 1.0 / (1.0 + np.exp(-g)) if sigmoid else g


def forward_stream(R, B, p):
    """(Rn, bound) for float64 operands; p: the keyword arguments of norm_residual."""
    F = R.shape[1]
    if p["post_norm"]:
        x, _, M = unit(B, p["kind"] == "layer", p["eps"])
        w, b = one(p["post_weight"], F), zero(p["post_bias"], F)
        v, M = w * x + b, np.abs(w) * M + np.abs(b)
    else:
        v, M = B, np.abs(B)
    g = p["scale"] * gate_values(p["gate"], p["gate_sigmoid"], R.shape)
    return R + g * v, K * U * (np.abs(R) + np.abs(g) * M)


def forward_norm(Rn, p):
    F = Rn.shape[1]
    x, _, M = unit(Rn, p["kind"] == "layer", p["eps"])
    w, b = one(p["pre_weight"], F), zero(p["pre_bias"], F)
    return w * x + b, K * U * (np.abs(w) * M + np.abs(b))


def backward(Rn, B, dZ, dRn, p):
    """{name: (value, bound)} of every gradient."""
    n, F = Rn.shape
    layer, eps = p["kind"] == "layer", p["eps"]
    mean = lambda a: a.mean(1, keepdims=True)  # noqa: E731

    def through(t, x, rho, M, mag):
        d = rho * (t - (mean(t) if layer else 0.0) - x * mean(t * x))
        return d, rho * (mag + (mean(mag) if layer else 0.0) + M * mean(mag * M))

    out = {}
    d = np.zeros_like(Rn) if dRn is None else dRn
    Md = np.abs(d)
    if dZ is not None:
        x, rho, M = unit(Rn, layer, eps)
        w = one(p["pre_weight"], F)
        out["pre_weight"] = ((dZ * x).sum(0), (np.abs(dZ) * M).sum(0))
        out["pre_bias"] = (dZ.sum(0), np.abs(dZ).sum(0))
        a, Ma = through(dZ * w, x, rho, M, np.abs(dZ * w))
        d, Md = d + a, Md + Ma
    out["R"] = (d, Md)
    if B is not None:
        x, rho, M = unit(B, layer, eps)
        w, b = one(p["post_weight"], F), zero(p["post_bias"], F)
        v, Mv = (w * x + b, np.abs(w) * M + np.abs(b)) if p["post_norm"] else (B, np.abs(B))
        g = gate_values(p["gate"], p["gate_sigmoid"], Rn.shape)
        slope = g * (1.0 - g) if p["gate_sigmoid"] else np.ones_like(g)
        dg, Mg = p["scale"] * d * v * slope, abs(p["scale"]) * Md * Mv * np.abs(slope)
        if p["gate"] is not None:
            axis = 0 if p["gate"].ndim == 1 else 1 if p["gate"].shape[1] == 1 and F != 1 else None
            if axis is None:
                out["gate"] = (dg, Mg)
            elif axis == 0:
                out["gate"] = (dg.sum(0), Mg.sum(0))
            else:
                out["gate"] = (dg.sum(1, keepdims=True), Mg.sum(1, keepdims=True))
        dv, Mdv = p["scale"] * d * g, abs(p["scale"]) * Md * np.abs(g)
        if p["post_norm"]:
            out["post_weight"] = ((dv * x).sum(0), (Mdv * M).sum(0))
            out["post_bias"] = (dv.sum(0), Mdv.sum(0))
            dv, Mdv = through(dv * w, x, rho, M, Mdv * np.abs(w))
        out["B"] = (dv, Mdv)
    return {k: (v, K_BACK * U * m) for k, (v, m) in out.items()}
