"""More operators of a deep GCN, trained on batches of graphs and served from 4 bits, as cases to be
timed and compared: their plain forms, and (where `own` is set) the library's calls.

Each case is a plain dict.  `kind` names the operator:

  group       Y = act(weight * (X - m) / sqrt(v + eps) + bias) with m and v over the nodes of a graph and
              the features of a group, for every graph of a batch (rows behind the last graph give 0)
  group_back  its gradients, for a gradient dY of Y
  clip        the norm of all gradients together, and the gradients scaled to a norm of max_norm at most
  step        the same norm, and W - lr * (clipped gradient)
  store       features brought into 4 bits (e2m1 with a power of two for each 32) and back
  mx          T = X W from 4-bit operands; "dynamic" cases bring X into 4 bits within the pass
"""
import math

import torch

own = False

DEV = "cuda:0"
BLOCK = 32


def listed():
    return [
        # one molecule-sized graph served: latency
        dict(name="group_one", kind="group", n=23, B=1, pad=0, F=64, G=8, act="silu", x="f32", y="bf16"),
        # a training batch of small graphs of 0 to some hundred nodes, padded behind the last
        dict(name="group_batch", kind="group", n=123457, B=4096, pad=577, F=128, G=8, act="relu", x="f32", y="f32"),
        # one large graph at the first layer's width, for a bfloat16 update
        dict(name="group_large", kind="group", n=1 << 21, B=1, pad=0, F=256, G=32, act="silu", x="f32", y="bf16"),
        # training on ragged graphs, an odd width
        dict(name="group_back_odd", kind="group_back", n=30011, B=300, pad=11, F=99, G=9, act="silu", x="bf16", y="f32"),
        # training on a few large graphs at the flagship's hidden width
        dict(name="group_back_large", kind="group_back", n=1 << 20, B=7, pad=0, F=128, G=16, act="relu", x="f32", y="f32"),
        # the two weights of a two-layer GCN, 256 -> 128 -> 64
        dict(name="clip_small", kind="clip", layers=1, F=128, F_in=256, F_out=64, vectors=0, bf16=False, max_norm=1.0),
        # a deep, wide GCN: matrices of 2,048 x 2,048, four vectors a layer, half of the layers in bfloat16
        dict(name="step_large", kind="step", layers=64, F=2048, F_in=528, F_out=47, vectors=4, bf16=True, max_norm=1.0),
        # the flagship's features (2^22 nodes of 256) kept in 4 bits and read back
        dict(name="store_large", kind="store", n=1 << 22, F=256, x="f32", out="bf16"),
        # one node served from 4 bits
        dict(name="mx_one", kind="mx", n=1, F_in=1024, F_out=256, dynamic=False, x="f32", out="f32"),
        # activations brought into 4 bits within the pass, ragged sizes (a last block of 16)
        dict(name="mx_dynamic", kind="mx", n=150001, F_in=400, F_out=136, dynamic=True, x="bf16", out="bf16"),
        # the flagship's first layer (256 -> 128, 2^22 nodes) on features kept in 4 bits
        dict(name="mx_large", kind="mx", n=1 << 22, F_in=256, F_out=128, dynamic=False, x="f32", out="f32"),
        # wide hidden layers, where the matrix unit counts
        dict(name="mx_wide", kind="mx", n=16384, F_in=4096, F_out=4096, dynamic=False, x="f32", out="bf16"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["group", "group", "group_back", "group_back", "clip", "step", "store", "mx", "mx", "mx"])
    x, y = rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"])
    if kind in ("group", "group_back"):
        G = rng.choice([1, 2, 4, 8, 16, 32, 3, 5, 9])
        D = log_int(1, 2048 // G)
        if rng.random() < 0.6:                      # most widths are multiples of 16
            D = max(1, D // 16 * 16)
        F = D * G
        n = log_int(1, max(1, min(1 << 21, (1 << (28 if kind == "group" else 27)) // F)))
        return dict(kind=kind, n=n, B=log_int(1, max(1, min(1 << 16, n))), pad=rng.choice([0, 0, n // 50]), F=F, G=G,
                    act=rng.choice(["none", "relu", "silu"]), x=x, y=y)
    if kind in ("clip", "step"):
        F = log_int(16, 2048)
        layers = log_int(1, max(1, min(96, (1 << 28) // (F * F))))
        return dict(kind=kind, layers=layers, F=F, F_in=log_int(16, 1024), F_out=log_int(2, 256), vectors=rng.choice([0, 1, 4]),
                    bf16=rng.random() < 0.4, max_norm=rng.choice([0.1, 1.0, 1e6]))
    if kind == "store":
        F = log_int(1, 4096)
        return dict(kind=kind, n=log_int(1, max(1, min(1 << 22, (1 << 29) // F))), F=F, x=x, out=y)
    F_in = log_int(16, 8192)
    if rng.random() < 0.7:
        F_in = max(32, F_in // 32 * 32)
    F_out = log_int(1, 4096)
    most = min((1 << 30) // max(F_in, 2 * F_out), (1 << 37) // (F_in * F_out))
    return dict(kind=kind, n=log_int(1, max(1, min(1 << 22, most))), F_in=F_in, F_out=F_out, dynamic=rng.random() < 0.4, x=x, out=y)


_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-5
CLIP_EPS = 1e-6
LR = 0.05


# ------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _prepare_group(c, g):
    n, B, F = c["n"], c["B"], c["F"]
    s = dict(c)
    # graphs of very different sizes: cuts at random places, some of them at the same place
    cuts = torch.sort(torch.randint(0, n - c["pad"] + 1, (B - 1,), generator=g, device=DEV)).values
    ends = torch.tensor([0, n - c["pad"]], device=DEV)
    s["ptr"] = torch.cat([ends[:1], cuts, ends[1:]]).to(torch.int32)
    # features that have a mean and a size of their own
    s["X"] = (_randn(g, n, F) * torch.exp(0.5 * _randn(g, F)) + 0.5 * _randn(g, F)).to(_TYPE[c["x"]])
    s["weight"], s["bias"] = 1.0 + 0.2 * _randn(g, F), 0.2 * _randn(g, F)
    if c["kind"] == "group_back":
        s["dY"] = (_randn(g, n, F) / math.sqrt(n)).to(_TYPE[c["y"]])
        s["stats"] = _group_stats(s)                # what the forward pass left
    return s


def _prepare_clip(c, g):
    s = dict(c)
    F = c["F"]
    shapes = [(c["F_in"], F)] + [(F, F)] * (c["layers"] - 1) + [(F, c["F_out"])]
    shapes += [(F,)] * (c["vectors"] * c["layers"])
    # gradients side by side in one piece of memory for each type; every other one is bfloat16
    kinds = [torch.bfloat16 if c["bf16"] and i % 2 else torch.float32 for i in range(len(shapes))]

    def views(dtypes):
        flat = {t: torch.empty(sum(math.prod(q) for q, k in zip(shapes, dtypes) if k == t), device=DEV, dtype=t) for t in set(dtypes)}
        pieces = {t: iter(flat[t].split([math.prod(q) for q, k in zip(shapes, dtypes) if k == t])) for t in flat}
        return flat, [next(pieces[k]).view(q) for q, k in zip(shapes, dtypes)]

    _, s["grads"] = views(kinds)
    for i, t in enumerate(s["grads"]):
        t.copy_(_randn(g, *t.shape) * (0.005 * (1 + i % 5)))
    if c["kind"] == "step":
        _, s["weights"] = views([torch.float32] * len(shapes))
        for t in s["weights"]:
            t.copy_(_randn(g, *t.shape) * 0.05)
        s["flat"], s["out"] = views([torch.float32] * len(shapes))
    else:
        s["flat"], s["out"] = views(kinds)
    return s


def _prepare_mx(c, g):
    s = dict(c)
    F = c["F"] if c["kind"] == "store" else c["F_in"]
    X = (_randn(g, c["n"], F).mul_(torch.exp(_randn(g, c["n"], 1)))).to(_TYPE[c["x"]])
    if c["kind"] == "store" or c["dynamic"]:
        s["X"] = X
    else:
        s["Xq"], s["sx"] = _packed(X)
    if c["kind"] == "mx":
        s["Wq"], s["sw"] = _packed((torch.rand(c["F_out"], F, generator=g, device=DEV) * 2 - 1) * math.sqrt(6.0 / (F + c["F_out"])))
    return s


def prepare(case, seed):
    g = _gen(seed)
    if case["kind"] in ("group", "group_back"):
        return _prepare_group(case, g)
    return _prepare_clip(case, g) if case["kind"] in ("clip", "step") else _prepare_mx(case, g)


# ------------------------------------------------------------------ one pass

def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    import paper_2609_01983_amd as dg

    kind = s["kind"]
    if kind in ("group", "group_back"):
        norm = dict(groups=s["G"], weight=s["weight"], bias=s["bias"], act=None if s["act"] == "none" else s["act"])
        if kind == "group":
            return dg.group_norm(s["X"], s["ptr"], eps=EPS, out_bf16=s["y"] == "bf16", **norm)
        return tuple(dg.group_norm_backward(s["X"], s["dY"], s["stats"], s["ptr"], **norm))
    if kind == "clip":
        _, norm = dg.clip_grads(s["grads"], s["max_norm"], eps=CLIP_EPS, out=s["out"])
        return {"norm": norm, **{str(t): f for t, f in s["flat"].items()}}
    if kind == "step":
        _, norm = dg.clipped_sgd(s["weights"], s["grads"], LR, s["max_norm"], eps=CLIP_EPS, out=s["out"])
        return {"norm": norm, **{str(t): f for t, f in s["flat"].items()}}
    if kind == "store":
        return dg.dequantize_mxfp4(*dg.quantize_mxfp4(s["X"]), s["F"], out_bf16=s["out"] == "bf16")
    Xq, sx = dg.quantize_mxfp4(s["X"]) if s["dynamic"] else (s["Xq"], s["sx"])
    return dg.update_mxfp4(Xq, sx, s["Wq"], s["sw"], out_bf16=s["out"] == "bf16")


def _plain(s):
    kind = s["kind"]
    if kind == "group":
        return _plain_group(s)
    if kind == "group_back":
        return _plain_group_back(s)
    if kind in ("clip", "step"):
        return _plain_clip(s)
    if kind == "store":
        q, k = _codes(s["X"])
        return _values(q, k)[:, :s["F"]].to(_TYPE[s["out"]])
    X = _values(*_codes(s["X"])) if s["dynamic"] else _unpacked(s["Xq"], s["sx"])
    return torch.matmul(X, _unpacked(s["Wq"], s["sw"]).t()).to(_TYPE[s["out"]])


def _graph_of(s):
    """The graph of every row (the last one's behind the last), and whether it is one of a graph."""
    row = torch.arange(s["n"], device=DEV)
    at = torch.searchsorted(s["ptr"].long(), row, right=True) - 1
    return at.clamp_(max=s["B"] - 1), (row < s["ptr"][-1]).unsqueeze(1)


def _over_graphs(s, v):
    """The sums of v (float64 [n, G]) over the rows of each graph."""
    c = torch.nn.functional.pad(torch.cumsum(v.t().contiguous(), 1), (1, 0))
    p = s["ptr"].long()
    return (c[:, p[1:]] - c[:, p[:-1]]).t()


def _members(s):
    p = s["ptr"].long()
    return ((p[1:] - p[:-1]).clamp(min=1) * (s["F"] // s["G"])).double().unsqueeze(1)


def _group_stats(s):
    """float64 [B, G, 2]: the mean and 1 / sqrt(variance + eps) of each graph and group."""
    X = s["X"].double().view(s["n"], s["G"], -1)
    m = _over_graphs(s, X.sum(2)) / _members(s)
    d = X - m[_graph_of(s)[0]].unsqueeze(2)
    v = _over_graphs(s, (d * d).sum(2)) / _members(s)
    return torch.stack([m, 1.0 / torch.sqrt(v + EPS)], 2)


def _unit(s, stats):
    """The normed features, in float64: a value next to 0 decides whether a ReLU passes it."""
    st = stats[_graph_of(s)[0]]
    u = (s["X"].double().view(s["n"], s["G"], -1) - st[:, :, :1]) * st[:, :, 1:]
    return u.reshape(s["n"], s["F"])


def _plain_group(s):
    stats = _group_stats(s)
    v = _unit(s, stats) * s["weight"] + s["bias"]
    if s["act"] == "relu":
        v = torch.where(v > 0, v, 0.0)
    if s["act"] == "silu":
        v = v / (1.0 + torch.exp(-v))
    return torch.where(_graph_of(s)[1], v, 0.0).to(_TYPE[s["y"]]), stats


def _plain_group_back(s):
    at, some = _graph_of(s)
    u = _unit(s, s["stats"])
    v = u * s["weight"] + s["bias"]
    d = torch.where(some, s["dY"].double(), 0.0)
    if s["act"] == "relu":
        d = torch.where(v > 0, d, 0.0)
    if s["act"] == "silu":
        q = 1.0 / (1.0 + torch.exp(-v))
        d = d * (q + v * q * (1.0 - q))
    t = d * s["weight"]
    mean = lambda a: _over_graphs(s, a.view(s["n"], s["G"], -1).sum(2)) / _members(s)  # noqa: E731
    wide = lambda a: a[at].unsqueeze(2).expand(-1, -1, s["F"] // s["G"]).reshape(s["n"], s["F"])  # noqa: E731
    dX = wide(s["stats"][:, :, 1]) * (t - wide(mean(t)) - u * wide(mean(t * u)))
    return torch.where(some, dX, 0.0).to(_TYPE[s["y"]]), (d * u).sum(0).float(), d.sum(0).float()


def _plain_clip(s):
    norm = torch.stack([t.double().square().sum() for t in s["grads"]]).sum().sqrt()
    f = torch.clamp(s["max_norm"] / (norm + CLIP_EPS), max=1.0)
    if s["kind"] == "step":
        new = [w - (LR * f).float() * t.float() for w, t in zip(s["weights"], s["grads"])]
    else:
        new = [(f.float() * t.float()).to(t.dtype) for t in s["grads"]]
    flat = {str(k): torch.cat([t.reshape(-1) for t in new if t.dtype == k]) for k in s["flat"]}
    return {"norm": norm.float().reshape(1), **flat}


def _blocks(F):
    return (F + BLOCK - 1) // BLOCK


def _codes(X):
    """(e2m1 values [n, blocks, 32], exponents [n, blocks, 1]): a block's scale is the least power of two
    that brings its largest to 7 = 0.875 * 2^3 at most (what is over 6 rounds to 6, as any other element
    by half a step at most)."""
    n, F = X.shape
    X = torch.nn.functional.pad(X.float(), (0, -F % BLOCK)).view(n, _blocks(F), BLOCK)
    amax = X.abs().amax(2, keepdim=True)
    m, e = torch.frexp(amax)
    k = torch.where(amax > 0, torch.where(m > 0.875, e - 2, e - 3).clamp(min=-127), 0)
    a = torch.ldexp(X, -k).abs()
    q = torch.where(a < 2, torch.round(2 * a) / 2, torch.where(a < 4, torch.round(a), 2 * torch.round(a / 2).clamp(max=3)))
    return torch.copysign(q, X), k


def _values(q, k):
    return torch.ldexp(q, k).flatten(1)


def _packed(X):
    """The 4-bit form of X: two codes a byte, the lower four bits first, [n, 16 blocks], and the exponents
    + 127, [n, blocks]."""
    pieces = [(slice(a, a + (1 << 18))) for a in range(0, X.shape[0], 1 << 18)]

    def one(x):
        q, k = _codes(x)
        a = q.abs()
        code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) + 8 * torch.signbit(q)
        return (code[..., ::2] + 16 * code[..., 1::2]).flatten(1).to(torch.uint8), (k.squeeze(2) + 127).to(torch.uint8)

    q, k = zip(*(one(X[p]) for p in pieces))
    return torch.cat(q), torch.cat(k)


def _unpacked(Q, scales):
    c = torch.stack([Q & 15, Q >> 4], 2).flatten(1).to(torch.int32)
    m = (c & 7).float()
    a = torch.where(m < 4, 0.5 * m, torch.where(m < 6, m - 2, 2 * m - 8))
    a = torch.where(c >= 8, -a, a).view(Q.shape[0], -1, BLOCK)
    return _values(a, scales.to(torch.int32).unsqueeze(2) - 127)


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("group", "group_back"):
        return _exact_group(case, s)
    return _exact_clip(case, s) if kind in ("clip", "step") else _exact_mx(case, s)


def _exact_group(c, s):
    """Forward by the definition; backward by automatic differentiation of it, some graphs at a time."""
    back = c["kind"] == "group_back"
    n, B, F, G = c["n"], c["B"], c["F"], c["G"]
    w, b = (s[k].double().requires_grad_(back) for k in ("weight", "bias"))
    ptr = s["ptr"].long().cpu().tolist()
    out = torch.zeros(n, F, dtype=torch.float64, device=DEV)
    stats, first = [], 0
    while first < B:
        last = first + 1                            # graphs first .. last - 1 of at most 2^26 elements, or one
        while last < B and (ptr[last + 1] - ptr[first]) * F <= 1 << 26:
            last += 1
        p = s["ptr"].long()[first:last + 1] - ptr[first]
        rows = slice(ptr[first], ptr[last])
        count = p.diff()
        at = torch.repeat_interleave(torch.arange(last - first, device=DEV), count)
        X = s["X"][rows].double().requires_grad_(back)
        x = X.unflatten(1, (G, F // G))
        size = (count.clamp(min=1) * (F // G)).unsqueeze(1)
        if last - first == 1:
            total = lambda a: a.sum((0, 2)).unsqueeze(0)  # noqa: E731
        else:
            total = lambda a: torch.zeros(last - first, G, dtype=torch.float64, device=DEV).index_add(0, at, a.sum(2))  # noqa: E731
        mean = total(x) / size
        off = x - mean[at].unsqueeze(2)
        inv = (total(off.pow(2)) / size + EPS).rsqrt()
        y = torch.addcmul(b, (off * inv[at].unsqueeze(2)).flatten(1), w)
        y = torch.relu(y) if c["act"] == "relu" else torch.nn.functional.silu(y) if c["act"] == "silu" else y
        if back:
            if X.numel():
                y.backward(s["dY"][rows].double())
                out[rows] = X.grad
        else:
            out[rows] = y
            stats.append(torch.stack([mean, inv], 2))
        first = last
    return (out, w.grad, b.grad) if back else (out, torch.cat(stats))


def _exact_clip(c, s):
    norm = math.sqrt(sum(float(torch.linalg.vector_norm(t, dtype=torch.float64)) ** 2 for t in s["grads"]))
    f = min(1.0, c["max_norm"] / (norm + CLIP_EPS))
    new = [(w.double() - LR * f * t.double()) if c["kind"] == "step" else f * t.double()
           for w, t in zip(s.get("weights", s["grads"]), s["grads"])]
    kinds = [torch.float32 if c["kind"] == "step" else t.dtype for t in s["grads"]]
    flat = {str(k): torch.cat([t.flatten() for t, q in zip(new, kinds) if q == k]) for k in s["flat"]}
    return {"norm": torch.tensor([norm], dtype=torch.float64), **flat}


def _rounded(X):
    """The values that X [n, F] has in 4 bits, by comparison with the middles between neighbours."""
    n, F = X.shape
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEV)
    out = torch.empty(n, F, dtype=torch.float64, device=DEV)
    for b in range(_blocks(F)):
        x = X[:, b * BLOCK:(b + 1) * BLOCK].double()
        big = x.abs().amax(1, keepdim=True)
        scale = torch.exp2(torch.ceil(torch.log2(torch.where(big > 0, big / 7, 1.0))).clamp(min=-127))
        a = (x / scale).abs()
        at = torch.zeros_like(a, dtype=torch.long)
        for j in range(7):                          # past the middle, or at it where the lower one is odd
            mid = (grid[j] + grid[j + 1]) / 2
            at += (a >= mid) if j % 2 else (a > mid)
        out[:, b * BLOCK:(b + 1) * BLOCK] = torch.copysign(grid[at] * scale, x)
    return out


def _exact_mx(c, s):
    half = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    table = torch.tensor(half + [-v for v in half], dtype=torch.float64, device=DEV)

    def decode(Q, scales):
        v = table[torch.stack([Q % 16, Q // 16], 2).long()].flatten(1)
        return v * torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, 1)

    F = c["F"] if c["kind"] == "store" else c["F_in"]
    step = max(1, (1 << 26) // (F + c.get("F_out", 0)))
    parts = [slice(a, min(c["n"], a + step)) for a in range(0, c["n"], step)]
    if c["kind"] == "store":
        return torch.cat([_rounded(s["X"][p]) for p in parts])
    W = decode(s["Wq"], s["sw"])[:, :F].t().contiguous()
    return torch.cat([(_rounded(s["X"][p]) if c["dynamic"] else decode(s["Xq"][p], s["sx"][p])[:, :F]) @ W for p in parts])


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = case
    kind = c["kind"]
    if kind in ("group", "group_back"):
        e = c["n"] * c["F"]
        x, y = _SIZE[c["x"]], _SIZE[c["y"]]
        fixed = 4 * (c["B"] + 1) + 8 * c["F"] + 16 * c["B"] * c["G"]
        if kind == "group":
            return {"bytes": e * (x + y) + fixed, "flops": 12 * e}
        return {"bytes": e * (x + 2 * y) + fixed + 8 * c["F"], "flops": 24 * e}
    if kind in ("clip", "step"):
        F = c["F"]
        sizes = [c["F_in"] * F] + [F * F] * (c["layers"] - 1) + [F * c["F_out"]] + [F] * (c["vectors"] * c["layers"])
        grads = [q * (2 if c["bf16"] and i % 2 else 4) for i, q in enumerate(sizes)]
        return {"bytes": sum(grads) + (8 * sum(sizes) if kind == "step" else sum(grads)) + 4, "flops": 4 * sum(sizes)}
    if kind == "store":
        return {"bytes": c["n"] * c["F"] * (_SIZE[c["x"]] + _SIZE[c["out"]]), "flops": 4 * c["n"] * c["F"]}
    n, F_in, F_out = c["n"], c["F_in"], c["F_out"]
    held = lambda rows: rows * _blocks(F_in) * 17  # noqa: E731
    x = n * F_in * _SIZE[c["x"]] if c["dynamic"] else held(n)
    return {"bytes": x + held(F_out) + n * F_out * _SIZE[c["out"]], "flops": 2 * n * F_in * F_out}
