"""The deep-GCN operators used together: a residual GCN trained from a teacher, forward and
backward, and served from 8-bit operands.  Every stage is checked on the inputs that the device
itself gave it, against float64 and with the bounds of that stage alone (normref.py, distillref.py,
1e-5 sum |a||x| for the aggregation, the products' float32 sums of bfloat16 operands), so the chain as a
whole is what its stages say."""
import threading

import numpy as np
import pytest
import torch

import distillref
import normref
import oracle
from graphgen import configs

pytestmark = pytest.mark.gpu

F, C, K, DEPTH = 64, 64, 8, 3


@pytest.fixture(scope="module")
def dg(device):
    import paper_2609_01983_amd as dg
    return dg


def host(t):
    return None if t is None else t.double().cpu().numpy()


def near(got, want, bound, what):
    g = host(got)
    bound = bound + (2.0 ** -8 * (np.abs(want) + bound) if got.dtype == torch.bfloat16 else 2.0 ** -24 * np.abs(want))
    bad = ~(np.abs(g - want) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} outside, first at {np.argwhere(bad)[0]}"


def rounded(t):
    return host(t.to(torch.bfloat16))


def product(got, X, W, what):
    """X W with both rounded to bfloat16: a float32 sum of at most 4,096 rows or columns' exact products in
    chains of 2^9 at most (a workgroup's rows, one k after another): 2^-14 of the magnitudes."""
    a, b = rounded(X), rounded(W)
    near(got, a @ b, 2.0 ** -14 * (np.abs(a) @ np.abs(b)), what)


class Net:
    """A stem, DEPTH blocks between norms, a head: R' = R + 0.5 gate post(A relu-less (Z W)), Z = pre(R')."""

    def __init__(self, dg, device):
        self.dg = dg
        g = self.g = configs.load_graph("c1")
        to = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)  # noqa: E731
        self.plan = dg.Plan(to(g.rowptr), to(g.col), to(g.val), seed=0, walks_per_node=4, walk_len=3)
        rng = np.random.default_rng(5)
        mat = lambda a, b: to((rng.standard_normal((a, b)) / np.sqrt(a)).astype(np.float32))  # noqa: E731
        vec = lambda about: to((about + 0.2 * rng.standard_normal(F)).astype(np.float32))  # noqa: E731
        self.X = to(rng.standard_normal((g.n, 32)).astype(np.float32))
        self.stem, self.head = mat(32, F), mat(F, C)
        self.W = [mat(F, F) for _ in range(DEPTH)]
        self.pre = [vec(1.0) for _ in range(DEPTH + 1)]
        self.post, self.gate = [vec(1.0) for _ in range(DEPTH)], [vec(0.0) for _ in range(DEPTH)]
        ids = np.argsort(rng.random((g.n, C)), axis=1)[:, :K].astype(np.int32)
        ids[::11] = -1
        ids[rng.random((g.n, K)) < 0.1] = -1
        self.ids, self.teacher = to(ids), to((2 * rng.standard_normal((g.n, K))).astype(np.float32))
        lab = rng.integers(0, C, g.n).astype(np.int32)
        lab[rng.random(g.n) < 0.6] = -1
        self.labels = to(lab)

    def spec(self, k):
        """The norms between block k - 1 (None before the first) and block k."""
        s = dict(pre_weight=self.pre[k])
        if k:
            s.update(post_weight=self.post[k - 1], gate=self.gate[k - 1], gate_sigmoid=True, scale=0.5)
        return s

    def reference(self, k):
        s = dict(post_norm=k > 0, post_weight=None, post_bias=None, pre_bias=None, gate=None, gate_sigmoid=False, scale=1.0,
                 kind="rms", eps=1e-5)
        s.update({n: host(v) if isinstance(v, torch.Tensor) else v for n, v in self.spec(k).items()})
        return s

    def forward(self, update):
        dg, s = self.dg, dict(T=[], B=[None], R=[], Z=[])
        s["R"].append(dg.update(self.X, self.stem))
        R, Z = dg.norm_residual(s["R"][0], norm_bf16=True, **self.spec(0))
        s["Z"].append(Z)
        for k in range(DEPTH):
            s["T"].append(update(Z, self.W[k]))
            s["B"].append(dg.spmm(self.plan, s["T"][-1]))
            R, Z = dg.norm_residual(R, s["B"][-1], norm_bf16=True, **self.spec(k + 1))
            s["R"].append(R)
            s["Z"].append(Z)
        s["T"].append(update(Z, self.head))
        s["Y"] = dg.spmm(self.plan, s["T"][-1])
        return s

    def backward(self, s):
        dg, n = self.dg, self.g.n
        b = dict(dT=[], dZ=[], dW=[], norm=[])
        b["G"], b["loss"] = dg.distill_xent(s["Y"], self.ids, self.teacher, self.labels, temperature=2.0,
                                            soft_scale=0.7 / n, hard_scale=0.3 / n)
        into, dR = b["G"], None
        for k in range(DEPTH, -1, -1):
            W = self.W[k] if k < DEPTH else self.head
            b["dT"].append(dg.spmm(self.plan, into, out_bf16=True))     # A is its own transpose
            b["dW"].append(dg.weight_grad(s["Z"][k], b["dT"][-1]))
            b["dZ"].append(dg.backward_data(b["dT"][-1], W))
            grads = dg.norm_residual_backward(s["R"][k], s["B"][k], b["dZ"][-1], dR, **self.spec(k))
            b["norm"].append(grads)
            dR, into = grads.R, grads.B
        b["dstem"] = dg.weight_grad(self.X, dR)
        return b


@pytest.fixture(scope="module")
def net(dg, device):
    return Net(dg, device)


def _check_spmm(net, X, Y, what):
    want, B = oracle.spmm(net.g, X.float().cpu().numpy())
    near(Y, want, 1e-5 * B, what)


def _check_norms(net, s):
    for k in range(DEPTH + 1):
        ref = net.reference(k)
        if k:
            near(s["R"][k], *normref.forward_stream(host(s["R"][k - 1]), host(s["B"][k]), ref), f"stream {k}")
        near(s["Z"][k], *normref.forward_norm(host(s["R"][k]), ref), f"norm {k}")


def test_training_step(net):
    s = net.forward(net.dg.update)
    b = net.backward(s)
    torch.cuda.synchronize()
    weights = net.W + [net.head]
    _check_norms(net, s)
    for k in range(DEPTH + 1):
        product(s["T"][k], s["Z"][k], weights[k], f"update {k}")
        _check_spmm(net, s["T"][k], s["B"][k + 1] if k < DEPTH else s["Y"], f"aggregation {k}")
    G, loss, bG, bl = distillref.distill(host(s["Y"]), net.ids.cpu().numpy(), host(net.teacher), net.labels.cpu().numpy(),
                                         2.0, float(np.float32(0.7 / net.g.n)), float(np.float32(0.3 / net.g.n)))
    near(b["G"], G, bG, "loss gradient")
    assert (np.abs(host(b["loss"]) - loss) <= bl).all()
    into, dR = b["G"], None
    for j, k in enumerate(range(DEPTH, -1, -1)):
        _check_spmm(net, into, b["dT"][j], f"gradient's aggregation {k}")
        product(b["dW"][j], s["Z"][k].t().contiguous(), b["dT"][j], f"weight gradient {k}")
        product(b["dZ"][j], b["dT"][j], weights[k].t().contiguous(), f"gradient's update {k}")
        want = normref.backward(host(s["R"][k]), host(s["B"][k]), host(b["dZ"][j]), host(dR), net.reference(k))
        got = b["norm"][j]
        for name in got._fields:
            if getattr(got, name) is not None:
                near(getattr(got, name), *want[name], f"d{name} {k}")
        dR, into = got.R, got.B
    product(b["dstem"], net.X.t().contiguous(), dR, "stem's gradient")
    # the same step again gives the same bits
    again = net.backward(net.forward(net.dg.update))
    assert torch.equal(again["dstem"], b["dstem"]) and torch.equal(again["loss"], b["loss"])


def test_serving_in_8_bits(net):
    dg = net.dg
    kept = {}

    def update(Z, W):
        if W.data_ptr() not in kept:                     # weights are laid out once
            kept[W.data_ptr()] = dg.quantize_weight_fp8(W)
        q, sx = dg.quantize_fp8(Z)
        T = dg.update_fp8(q, sx, *kept[W.data_ptr()])
        Wq, sw = kept[W.data_ptr()]
        a = host(q) * np.repeat(host(sx), 128, 1)[:, :F]
        w = host(Wq) * np.repeat(np.repeat(host(sw), 128, 1)[:, :F], 128, 0)[:W.shape[1]]
        near(T, a @ w.T, 2 * 2.0 ** -24 * 144 * (np.abs(a) @ np.abs(w).T), "8-bit update")
        # a node by itself: the same product, summed in its own order
        one = dg.update_fp8(q[7:8].contiguous(), sx[7:8].contiguous(), Wq, sw)
        near(one, (a @ w.T)[7:8], 2 * 2.0 ** -24 * 144 * (np.abs(a) @ np.abs(w).T)[7:8], "8-bit update of one node")
        return T

    s = net.forward(update)
    torch.cuda.synchronize()
    _check_norms(net, s)
    for k in range(DEPTH + 1):
        _check_spmm(net, s["T"][k], s["B"][k + 1] if k < DEPTH else s["Y"], f"aggregation {k}")


def test_two_threads_on_two_streams(net, device):
    """Calls of two host threads that overlap, each on its own stream with its own outputs."""
    dg = net.dg
    s = net.forward(dg.update)
    dZ = torch.randn(net.g.n, F, device=device)
    want_n = dg.norm_residual_backward(s["R"][1], s["B"][1], dZ, None, **net.spec(1))
    want_d = dg.distill_xent(s["Y"], net.ids, net.teacher, net.labels, soft_scale=0.1, hard_scale=0.1)
    torch.cuda.synchronize()
    wrong = []

    def work(which):
        stream = torch.cuda.Stream(device)
        with torch.cuda.stream(stream):
            for _ in range(20):
                if which:
                    got = dg.norm_residual_backward(s["R"][1], s["B"][1], dZ, None, **net.spec(1))
                    same = all(x is None or torch.equal(x, y) for x, y in zip(got, want_n))
                else:
                    G, loss = dg.distill_xent(s["Y"], net.ids, net.teacher, net.labels, soft_scale=0.1, hard_scale=0.1)
                    same = torch.equal(G, want_d[0]) and torch.equal(loss, want_d[1])
                if not same:
                    wrong.append(which)
            stream.synchronize()

    threads = [threading.Thread(target=work, args=(k % 2,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
