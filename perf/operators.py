"""The operators of a deep GCN that is trained from a teacher and served in 8 bits, as cases to
be timed and compared: their plain forms, and (where `own` is set) the library's calls.

Each case is a plain dict.  `kind` names the operator:

  norm      R' = R + scale * gate * post(B) and Z = pre(R'): the norms after and before a block
            (RMS or layer norm) with the block's gate and residual scale
  norm_back its gradients, for gradients dZ of Z and dR' of R'
  distill   the loss against a teacher's top logits (temperature, renormalised over the kept
            ones) with the labels' cross-entropy, and its gradient
  fp8       T = X W from e4m3 operands with a float32 scale for each block of 128; "dynamic"
            cases quantise X within the pass, the others have stored features
"""
import math

import torch

own = False

DEV = "cuda:0"
BLOCK = 128


def listed():
    return [
        # one node served: the norm before the first block of a bfloat16 model
        dict(name="norm_one", kind="norm", n=1, F=256, layer=False, post=False, pre=True, block=False,
             gate="none", sigmoid=False, act="bf16", stream="f32", z="bf16"),
        # the smallest workload's graph (4,096 nodes): layer norms, a learned gate for each feature
        dict(name="norm_small", kind="norm", n=4096, F=64, layer=True, post=True, pre=True, block=True,
             gate="col", sigmoid=False, act="f32", stream="f32", z="f32"),
        # a block of a large graph between its aggregation (float32) and the next update (bfloat16)
        dict(name="norm_large", kind="norm", n=1 << 21, F=256, layer=False, post=True, pre=True, block=True,
             gate="col", sigmoid=False, act="f32", stream="f32", z="bf16"),
        # training a small graph: ragged rows, an odd width, a gate for each element through a sigmoid
        dict(name="norm_back_odd", kind="norm_back", n=20001, F=99, layer=True, post=True, pre=True, block=True,
             gate="full", sigmoid=True, act="bf16", stream="f32", grad="f32"),
        # training at the flagship's hidden width on a million nodes
        dict(name="norm_back_large", kind="norm_back", n=1 << 20, F=128, layer=False, post=True, pre=True,
             block=True, gate="col", sigmoid=False, act="f32", stream="f32", grad="f32"),
        # wide hidden states, everything in bfloat16
        dict(name="norm_back_wide", kind="norm_back", n=8191, F=4096, layer=False, post=True, pre=True,
             block=True, gate="none", sigmoid=False, act="bf16", stream="bf16", grad="bf16"),
        # a small graph's last layer: 47 classes, eight kept logits a node, 30% of the nodes labelled
        dict(name="distill_small", kind="distill", n=30007, C=47, K=8, T=2.0, hard=True, y="f32", g="f32"),
        # the flagship's last layer: 2^22 nodes of 64 classes
        dict(name="distill_large", kind="distill", n=1 << 22, C=64, K=16, T=4.0, hard=True, y="f32", g="f32"),
        # a vocabulary of classes, many rows, bfloat16 logits and gradients
        dict(name="distill_vocab", kind="distill", n=4095, C=131072, K=64, T=1.0, hard=True, y="bf16", g="bf16"),
        # one node served from 8-bit features
        dict(name="fp8_one", kind="fp8", n=1, F_in=1024, F_out=256, dynamic=False, x="f32", out="f32"),
        # activations quantised within the pass, ragged sizes
        dict(name="fp8_dynamic", kind="fp8", n=200003, F_in=528, F_out=200, dynamic=True, x="bf16", out="bf16"),
        # the flagship's first layer (256 -> 128, 2^22 nodes) on features kept in 8 bits
        dict(name="fp8_large", kind="fp8", n=1 << 22, F_in=256, F_out=128, dynamic=False, x="f32", out="f32"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["norm", "norm_back", "distill", "fp8"])
    if kind in ("norm", "norm_back"):
        F = log_int(8, 8192)
        if rng.random() < 0.6:                      # most widths are multiples of 16
            F = max(16, F // 16 * 16)
        most = 1 << 28 if kind == "norm" else 1 << 27
        n = log_int(1, max(1, min(1 << 21, most // F)))
        c = dict(kind=kind, n=n, F=F, layer=rng.random() < 0.4, post=rng.random() < 0.7, pre=rng.random() < 0.85,
                 block=True, gate=rng.choice(["none", "col", "col", "row", "full"]), act=rng.choice(["f32", "bf16"]),
                 stream=rng.choice(["f32", "f32", "bf16"]))
        c["sigmoid"] = c["gate"] != "none" and rng.random() < 0.3
        if kind == "norm":
            c["z"] = rng.choice(["f32", "bf16"])
            if rng.random() < 0.2:
                c.update(block=False, post=False, pre=True, gate="none", sigmoid=False)
        else:
            c["grad"] = rng.choice(["f32", "f32", "bf16"])
        return c
    if kind == "distill":
        C = log_int(2, 200000)
        K = min(C, log_int(1, 256))
        n = log_int(1, max(1, min(1 << 22, (1 << 28) // (C + 2 * K))))
        return dict(kind=kind, n=n, C=C, K=K, T=rng.choice([1.0, 2.0, 3.5]),
                    hard=rng.random() < 0.6, y=rng.choice(["f32", "bf16"]), g=rng.choice(["f32", "bf16"]))
    F_in = 16 * log_int(2, 64)
    F_out = log_int(16, 1024)
    n = log_int(1, min(1 << 22, (1 << 30) // max(F_in, 2 * F_out)))
    return dict(kind=kind, n=n, F_in=F_in, F_out=F_out, dynamic=rng.random() < 0.4, x=rng.choice(["f32", "bf16"]),
                out=rng.choice(["f32", "bf16"]))


_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-5
SCALE = 0.7


# ------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _prepare_norm(c, g):
    n, F = c["n"], c["F"]
    s = {k: c[k] for k in c if k != "gate"}
    # a stream that has grown over some blocks, with rows of different sizes and a few hot features
    size = torch.exp(0.5 * _randn(g, n, 1))
    hot = 1.0 + 4.0 * (torch.rand(F, generator=g, device=DEV) < 0.02)
    s["R"] = (_randn(g, n, F) * size * hot + 0.1).to(_TYPE[c["stream"]])
    s["B"] = (_randn(g, n, F).mul_(torch.exp(0.5 * _randn(g, n, 1))).add_(0.2)).to(_TYPE[c["act"]]) if c["block"] else None
    vec = lambda about: about + 0.2 * _randn(g, F)  # noqa: E731
    s["post_weight"] = vec(1.0) if c["post"] else None
    s["post_bias"] = vec(0.0) if c["post"] and c["layer"] else None
    s["pre_weight"] = vec(1.0) if c["pre"] else None
    s["pre_bias"] = vec(0.0) if c["pre"] and c["layer"] else None
    shape = {"none": None, "col": (F,), "row": (n, 1), "full": (n, F)}[c["gate"]]
    s["gate"] = None if shape is None else _randn(g, *shape).mul_(0.5).add_(0.5)
    if c["gate"] == "full":
        s["gate"] = s["gate"].to(_TYPE[c["act"]])
    if c["kind"] == "norm_back":
        t = _TYPE[c["grad"]]
        s["dZ"] = (_randn(g, n, F) / math.sqrt(n)).to(t) if c["pre"] else None
        s["dRn"] = (_randn(g, n, F) / math.sqrt(n)).to(_TYPE[c["stream"]])
    return s


def _prepare_distill(c, g):
    n, C, K = c["n"], c["C"], c["K"]
    s = dict(c)
    s["Y"] = _randn(g, n, C).mul_(2.0).to(_TYPE[c["y"]])
    # distinct classes, one of each of K strata; the teacher's logits fall along the row
    k = (torch.arange(K, device=DEV) + torch.randint(0, K, (n, 1), generator=g, device=DEV)) % K
    low, high = k * C // K, (k + 1) * C // K
    ids = low + (torch.rand(n, K, generator=g, device=DEV) * (high - low)).long()
    t = 8.0 - torch.cumsum(torch.rand(n, K, generator=g, device=DEV) * (4.0 / math.sqrt(K)), 1)
    # a tenth of the rows keep fewer entries, 5% of the rows have no teacher at all
    kept = torch.where(torch.rand(n, 1, generator=g, device=DEV) < 0.1,
                       torch.randint(0, K + 1, (n, 1), generator=g, device=DEV), K)
    kept[torch.rand(n, 1, generator=g, device=DEV) < 0.05] = 0
    ids = torch.where(torch.arange(K, device=DEV) < kept, torch.minimum(ids, high - 1), -1)
    s["ids"], s["teacher"] = ids.to(torch.int32), t
    labels = torch.randint(0, C, (n,), generator=g, device=DEV)
    labels[torch.rand(n, generator=g, device=DEV) >= 0.3] = -1
    s["labels"] = labels.to(torch.int32) if c["hard"] else None
    s["soft_scale"], s["hard_scale"] = 0.7 / n, 0.3 / max(1.0, 0.3 * n)
    return s


def _blocks(F):
    return (F + BLOCK - 1) // BLOCK


def _pad(x, dim):
    """x with zeros up to whole blocks along dim."""
    more = -x.shape[dim] % BLOCK
    shape = list(x.shape)
    shape[dim] = more
    return torch.cat([x, x.new_zeros(shape)], dim) if more else x


def _stored(x, amax, expand):
    """(e4m3 values, float32 scales): the largest of a block at e4m3's largest, 448."""
    scale = torch.where(amax > 0, amax / 448.0, torch.ones_like(amax))
    return (x / expand(scale)).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn), scale


def _prepare_fp8(c, g):
    n, F_in, F_out = c["n"], c["F_in"], c["F_out"]
    s = dict(c)
    X = _randn(g, n, F_in).mul_(torch.exp(_randn(g, n, 1)))
    W = (torch.rand(F_out, F_in, generator=g, device=DEV) * 2 - 1) * math.sqrt(6.0 / (F_in + F_out))
    cols = lambda t: t.repeat_interleave(BLOCK, 1)[:, :F_in]  # noqa: E731
    if c["dynamic"]:
        s["X"] = X.to(_TYPE[c["x"]])
    else:
        amax = _pad(X, 1).abs().reshape(n, _blocks(F_in), BLOCK).amax(2)
        s["Xq"], s["sx"] = _stored(X, amax, cols)
    Wp = _pad(_pad(W, 0), 1).abs().reshape(_blocks(F_out), BLOCK, _blocks(F_in), BLOCK)
    s["Wq"], s["sw"] = _stored(W, Wp.amax((1, 3)), lambda t: cols(t).repeat_interleave(BLOCK, 0)[:F_out])
    return s


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    if kind in ("norm", "norm_back"):
        return _prepare_norm(case, g)
    return _prepare_distill(case, g) if kind == "distill" else _prepare_fp8(case, g)


# ------------------------------------------------------------------ one pass

def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    import paper_2609_01983_amd as dg

    kind = s["kind"]
    if kind in ("norm", "norm_back"):
        block = dict(post_norm=s["post"], post_weight=s["post_weight"], post_bias=s["post_bias"], gate=s["gate"],
                     gate_sigmoid=s["sigmoid"], scale=SCALE, pre_norm=s["pre"], pre_weight=s["pre_weight"],
                     pre_bias=s["pre_bias"], kind="layer" if s["layer"] else "rms", eps=EPS)
        if kind == "norm":
            Rn, Z = dg.norm_residual(s["R"], s["B"], norm_bf16=s["z"] == "bf16", **block)
            return (Rn if s["block"] else None, Z)
        # the stream after the block is what the forward pass left: here the state's R stands for it
        return tuple(dg.norm_residual_backward(s["R"], s["B"], s["dZ"], s["dRn"],
                                               grad_bf16=s["grad"] == "bf16", **block))
    if kind == "distill":
        return dg.distill_xent(s["Y"], s["ids"], s["teacher"], s["labels"], temperature=s["T"],
                               soft_scale=s["soft_scale"], hard_scale=s["hard_scale"], grad_bf16=s["g"] == "bf16")
    Xq, sx = dg.quantize_fp8(s["X"]) if s["dynamic"] else (s["Xq"], s["sx"])
    return dg.update_fp8(Xq, sx, s["Wq"], s["sw"], out_bf16=s["out"] == "bf16")


def _plain(s):
    kind = s["kind"]
    if kind == "norm":
        return _plain_norm(s)
    if kind == "norm_back":
        return _plain_norm_back(s)
    return _plain_distill(s) if kind == "distill" else _plain_fp8(s)


def _unit(x, layer):
    """The rows of x centred (layer norm) and divided by their root mean square, and 1 / that."""
    c = x - x.mean(1, keepdim=True) if layer else x
    r = 1.0 / torch.sqrt((c * c).mean(1, keepdim=True) + EPS)
    return c * r, r


def _gate_of(s):
    """The gate as it multiplies; its logits' derivative."""
    if s["gate"] is None:
        return None, None
    g = s["gate"].float()
    if not s["sigmoid"]:
        return g, None
    g = 1.0 / (1.0 + torch.exp(-g))
    return g, g * (1.0 - g)


def _affine(u, w, b):
    u = u if w is None else u * w
    return u if b is None else u + b


def _plain_norm(s):
    R = s["R"].float()
    Rn = None
    if s["block"]:
        v = s["B"].float()
        if s["post"]:
            v = _affine(_unit(v, s["layer"])[0], s["post_weight"], s["post_bias"])
        g, _ = _gate_of(s)
        v = v if g is None else v * g
        Rn = (R + SCALE * v).to(_TYPE[s["stream"]])
        R = Rn.float()
    Z = None
    if s["pre"]:
        Z = _affine(_unit(R, s["layer"])[0], s["pre_weight"], s["pre_bias"]).to(_TYPE[s["z"]])
    return (Rn, Z)


def _unit_back(t, u, r, layer):
    d = t - u * (t * u).mean(1, keepdim=True)
    return r * (d - t.mean(1, keepdim=True) if layer else d)


def _plain_norm_back(s):
    grad, stream = _TYPE[s["grad"]], _TYPE[s["stream"]]
    d = s["dRn"].float()
    dw2 = db2 = dw1 = db1 = dgate = None
    if s["pre"]:
        u, r = _unit(s["R"].float(), s["layer"])
        dZ = s["dZ"].float()
        dw2 = (dZ * u).double().sum(0).float()
        db2 = dZ.double().sum(0).float() if s["pre_bias"] is not None else None
        d = d + _unit_back(dZ * s["pre_weight"], u, r, s["layer"])
    dR = d.to(stream)
    v = s["B"].float()
    if s["post"]:
        u1, r1 = _unit(v, s["layer"])
        v = _affine(u1, s["post_weight"], s["post_bias"])
    g, slope = _gate_of(s)
    dv = SCALE * d
    if g is not None:
        dg = dv * v
        dg = dg if slope is None else dg * slope
        if s["gate"].dim() == 1:
            dgate = dg.double().sum(0).float()
        else:
            dgate = dg.to(grad) if s["gate"].shape == dg.shape else dg.double().sum(1, keepdim=True).float()
        dv = dv * g
    if s["post"]:
        dw1 = (dv * u1).double().sum(0).float()
        db1 = dv.double().sum(0).float() if s["post_bias"] is not None else None
        dv = _unit_back(dv * s["post_weight"], u1, r1, s["layer"])
    return (dR, dv.to(grad), dgate, dw1, db1, dw2, db2)


def _plain_distill(s):
    Y, T = s["Y"].float(), s["T"]
    C = Y.shape[1]
    ok = (s["ids"] >= 0) & (s["ids"] < C)
    ids = torch.where(ok, s["ids"], 0).long()
    t = torch.where(ok, s["teacher"] / T, -math.inf)
    taught = ok.any(1, keepdim=True)
    t = t - torch.where(taught, t.amax(1, keepdim=True), 0.0)
    e = torch.exp(t)
    total = torch.where(taught, e.sum(1, keepdim=True), 1.0)
    p = e / total
    x = Y / T
    x = x - x.amax(1, keepdim=True)
    ex = torch.exp(x)
    sx = ex.sum(1, keepdim=True)
    terms = p * (t - torch.log(total) - torch.gather(x, 1, ids) + torch.log(sx))
    soft = s["soft_scale"] * T * T * torch.where(p > 0, terms, 0.0).double().sum()
    G = (s["soft_scale"] * T) * torch.where(taught, ex / sx, 0.0)
    G.scatter_add_(1, ids, (-s["soft_scale"] * T) * p)
    hard = torch.zeros_like(soft)
    if s["labels"] is not None:
        labeled = (s["labels"] >= 0) & (s["labels"] < C)
        at = torch.where(labeled, s["labels"], 0).long()[:, None]
        x = Y - Y.amax(1, keepdim=True)
        ex = torch.exp(x)
        sx = ex.sum(1, keepdim=True)
        hard = s["hard_scale"] * torch.where(labeled[:, None], torch.log(sx) - torch.gather(x, 1, at), 0.0).double().sum()
        G += s["hard_scale"] * torch.where(labeled[:, None], ex / sx, 0.0)
        G.scatter_add_(1, at, torch.where(labeled[:, None], -s["hard_scale"], 0.0))
    return (G.to(_TYPE[s["g"]]), torch.stack([soft + hard, soft, hard]).float())


def _quantised(X):
    """(e4m3 values, float32 scales): a block's scale is the least power of two that brings its
    largest to 448 = 0.875 * 2^9 at most."""
    n, F = X.shape
    amax = _pad(X.float(), 1).abs().reshape(n, _blocks(F), BLOCK).amax(2)
    m, e = torch.frexp(amax)
    k = torch.where(m > 0.875, e - 8, e - 9).clamp_(min=-126)
    scale = torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), k), 1.0)
    return (X.float() / scale.repeat_interleave(BLOCK, 1)[:, :F]).to(torch.float8_e4m3fn), scale


def _plain_fp8(s):
    Xq, sx = _quantised(s["X"]) if s["dynamic"] else (s["Xq"], s["sx"])
    F_out, F_in = s["Wq"].shape
    X = Xq.float() * sx.repeat_interleave(BLOCK, 1)[:, :F_in]
    W = s["Wq"].float() * s["sw"].repeat_interleave(BLOCK, 1)[:, :F_in].repeat_interleave(BLOCK, 0)[:F_out]
    return torch.matmul(X, W.t()).to(_TYPE[s["out"]])


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("norm", "norm_back"):
        return _exact_norm(case, s)
    return _exact_distill(s) if kind == "distill" else _exact_fp8(case, s)


def _chunks(n, width):
    step = max(1, (1 << 27) // max(1, width))
    return [slice(a, min(n, a + step)) for a in range(0, n, step)]


def _exact_norm(c, s):
    """Forward by the definition; backward by automatic differentiation of it, both in float64."""
    back = c["kind"] == "norm_back"
    leaf = lambda t: None if t is None else t.double().requires_grad_(back)  # noqa: E731
    w1, b1, w2, b2 = (leaf(s[k]) for k in ("post_weight", "post_bias", "pre_weight", "pre_bias"))
    shared = leaf(s["gate"]) if c["gate"] == "col" else None

    def normed(x, w, b):
        if c["layer"]:
            x = x - x.sum(-1, keepdim=True) / c["F"]
        return torch.addcmul(b if b is not None else torch.zeros_like(w), x / (x.pow(2).sum(-1, keepdim=True) / c["F"] + EPS).sqrt(), w)

    parts = []
    for at in _chunks(c["n"], c["F"]):
        R, B = leaf(s["R"][at]), leaf(s["B"][at]) if c["block"] else None
        gate = shared if c["gate"] == "col" else leaf(s["gate"][at]) if s["gate"] is not None else None
        joined = None
        if B is not None:
            v = normed(B, w1, b1) if c["post"] else B
            if gate is not None:
                v = v * (torch.sigmoid(gate) if c["sigmoid"] else gate)
            # in the backward pass the state's R is the stream after the block
            joined = SCALE * v if back else R + SCALE * v
        if not back:
            Rn = None if joined is None else joined
            # the next norm takes the stream as it is stored
            held = R if Rn is None else Rn.to(_TYPE[c["stream"]]).double() if c["stream"] == "bf16" else Rn
            parts.append((Rn, normed(held, w2, b2) if c["pre"] else None))
            continue
        dRn = s["dRn"][at].double()
        if c["pre"]:
            normed(R, w2, b2).backward(s["dZ"][at].double())
            dRn = dRn + R.grad
        joined.backward(dRn)
        parts.append((dRn, B.grad, gate.grad if c["gate"] in ("row", "full") else None))
    rows = [None if p[0] is None else torch.cat(p) for p in zip(*parts)]
    if not back:
        return tuple(rows)
    sums = [None if t is None else t.grad for t in (w1, b1, w2, b2)]
    return (rows[0], rows[1], shared.grad if shared is not None else rows[2], *sums)


def _exact_distill(s):
    n, C = s["Y"].shape
    T, a, h = s["T"], s["soft_scale"], s["hard_scale"]
    G, soft, hard = [], 0.0, 0.0
    for at in _chunks(n, C):
        Y = s["Y"][at].double()
        m = Y.shape[0]
        ids = s["ids"][at].long()
        valid = (ids >= 0) & (ids < C)
        logits = (s["teacher"][at].double() / T).masked_fill(~valid, -math.inf)
        row = valid.any(1)
        P = torch.zeros(m, C + 1, dtype=torch.float64, device=DEV)
        P.scatter_add_(1, torch.where(valid, ids, C), torch.nan_to_num(torch.softmax(logits, 1), nan=0.0))
        P = P[:, :C]
        lq = torch.log_softmax(Y / T, 1)
        pk = torch.where(row[:, None], torch.softmax(logits, 1), 0.0)
        kl = torch.special.xlogy(pk, pk).sum(1) - (P * lq).sum(1)
        soft += float(kl[row].sum())
        g = a * T * (lq.exp() - P) * row[:, None]
        if s["labels"] is not None:
            lab = s["labels"][at].long()
            has = (lab >= 0) & (lab < C)
            l1 = torch.log_softmax(Y, 1)
            pick = lab.clamp(0, C - 1).unsqueeze(1)
            hard -= float(l1.gather(1, pick).squeeze(1)[has].sum())
            one = torch.zeros_like(Y).scatter_(1, pick, 1.0)
            g = g + h * (l1.exp() - one) * has[:, None]
        G.append(g)
    soft, hard = a * T * T * soft, h * hard
    return (torch.cat(G), torch.tensor([soft + hard, soft, hard], dtype=torch.float64))


def _exact_fp8(c, s):
    n, F_in, F_out = c["n"], c["F_in"], c["F_out"]
    W = s["Wq"].double()
    out = []
    for at in _chunks(n, 4 * max(F_in, F_out)):
        T = 0.0
        for b in range(_blocks(F_in)):
            k = slice(b * BLOCK, min(F_in, (b + 1) * BLOCK))
            if c["dynamic"]:
                X = s["X"][at, k].double()
                big = X.abs().amax(1, keepdim=True)
                scale = torch.exp2(torch.ceil(torch.log2(torch.where(big > 0, big / 448.0, 1.0))))
                X, sx = (X / scale).float().to(torch.float8_e4m3fn).double(), scale
            else:
                X, sx = s["Xq"][at, k].double(), s["sx"][at, b:b + 1].double()
            sw = s["sw"][:, b].double().repeat_interleave(BLOCK)[:F_out]
            T = T + (X @ W[:, k].t()) * sx * sw
        out.append(T)
    return torch.cat(out)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = case
    kind = c["kind"]
    if kind in ("norm", "norm_back"):
        e = c["n"] * c["F"]
        act, stream = _SIZE[c["act"]], _SIZE[c["stream"]]
        gate = {"none": 0, "col": 4 * c["F"], "row": 4 * c["n"], "full": e * act}[c["gate"]]
        vectors = 4 * c["F"] * (c["post"] + c["pre"]) * (2 if c["layer"] else 1)
        if kind == "norm":
            moved = e * stream + (e * (act + stream) if c["block"] else 0) + (e * _SIZE[c["z"]] if c["pre"] else 0)
            return {"bytes": moved + gate + vectors, "flops": 16 * e}
        grad = _SIZE[c["grad"]]
        moved = e * (act + 2 * stream + grad) + (e * (stream + grad) if c["pre"] else 0)
        back = {"none": 0, "col": 4 * c["F"], "row": 4 * c["n"], "full": e * grad}[c["gate"]]
        return {"bytes": moved + gate + back + 2 * vectors, "flops": 30 * e}
    if kind == "distill":
        e = c["n"] * c["C"]
        # Y is read on rows that are taught or labelled (95% and more); the entries and labels of all
        return {"bytes": e * (_SIZE[c["y"]] + _SIZE[c["g"]]) + 8 * c["n"] * c["K"] + (4 * c["n"] if c["hard"] else 0),
                "flops": (12 if c["hard"] else 7) * e}
    n, F_in, F_out = c["n"], c["F_in"], c["F_out"]
    x = n * F_in * _SIZE[c["x"]] if c["dynamic"] else n * (F_in + 4 * _blocks(F_in))
    return {"bytes": x + F_in * F_out + 4 * _blocks(F_in) * _blocks(F_out) + n * F_out * _SIZE[c["out"]],
            "flops": 2 * n * F_in * F_out}
