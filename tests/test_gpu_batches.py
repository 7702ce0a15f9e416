"""The operators over batches used together: a GCN on a batch of graphs, trained with clipped steps and served from 4-bit
operands.  Every stage is checked on the inputs that the device itself gave it, against float64 and with the bounds of that
stage alone (groupref.py; 1e-5 sum |a||x| for the aggregation; the products' float32 sums; a rounding for the step)."""
from concurrent.futures import ThreadPoolExecutor

import math

import numpy as np
import pytest
import torch

import groupref
import oracle
from graphgen import csr

pytestmark = pytest.mark.gpu

F_IN, F, C, G = 32, 64, 32, 8
EPS = 1e-5


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
    """X W with both rounded to bfloat16: float32 sums of exact products in chains of 2^9 at most: 2^-14 of the magnitudes."""
    a, b = rounded(X), rounded(W)
    near(got, a @ b, 2.0 ** -14 * (np.abs(a) @ np.abs(b)), what)


class Batch:
    """Graphs of 1 to some hundred nodes side by side (one without nodes), each connected at random, and rows of padding behind
    the last; every row has a self-loop."""

    def __init__(self, dg, device):
        self.dg = dg
        rng = np.random.default_rng(12)
        sizes = [17, 1, 0, 40, 300, 2, 33, 128, 5, 700, 1, 64, 90, 31]
        self.ptr = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
        used = int(self.ptr[-1])
        self.n = n = used + 24
        pairs = []
        for lo, hi in zip(self.ptr[:-1], self.ptr[1:]):
            if hi - lo > 1:
                e = rng.integers(lo, hi, (4 * (hi - lo), 2))
                pairs.append(e[e[:, 0] != e[:, 1]])
        e = np.concatenate(pairs)
        e = np.unique(np.concatenate([e, e[:, ::-1], np.stack([np.arange(n)] * 2, 1)]), axis=0)
        rowptr = np.concatenate([[0], np.cumsum(np.bincount(e[:, 0], minlength=n))]).astype(np.int32)
        deg = np.diff(rowptr).astype(np.float64)
        val = (1.0 / np.sqrt(deg[e[:, 0]] * deg[e[:, 1]])).astype(np.float32)
        self.g = csr.Graph(n, rowptr, e[:, 1].astype(np.int32), val)
        to = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)  # noqa: E731
        self.plan = dg.Plan(to(rowptr), to(e[:, 1].astype(np.int32)), to(val), seed=0, walks_per_node=4, walk_len=3)
        self.X, self.dptr = to(rng.standard_normal((n, F_IN)).astype(np.float32)), to(self.ptr)
        mat = lambda a, b: to((rng.standard_normal((a, b)) / np.sqrt(a)).astype(np.float32))  # noqa: E731
        self.W = [mat(F_IN, F), mat(F, F), mat(F, C)]
        self.vec = [to((1 - k % 2 + 0.2 * rng.standard_normal(F)).astype(np.float32)) for k in range(4)]       # weight, bias, weight, bias
        lab = rng.integers(0, C, n).astype(np.int32)
        lab[used:] = -1
        self.labels, self.scale = to(lab), 1.0 / used

    def norm(self, k):
        return dict(groups=G, weight=self.vec[2 * k], bias=self.vec[2 * k + 1], act=("silu", "relu")[k])

    def forward(self, update):
        dg, s = self.dg, dict(H=[self.X], T=[], P=[], stats=[])
        for k in range(2):
            s["T"].append(update(s["H"][-1], self.W[k]))
            s["P"].append(dg.spmm(self.plan, s["T"][-1]))
            H, stats = dg.group_norm(s["P"][-1], self.dptr, out_bf16=True, eps=EPS, **self.norm(k))
            s["H"].append(H)
            s["stats"].append(stats)
        s["Y"] = update(s["H"][-1], self.W[2])
        return s

    def backward(self, s):
        dg, b = self.dg, dict(dH=[], norm=[], dT=[], dW=[])
        b["G"], b["loss"] = dg.softmax_xent(s["Y"], self.labels, self.scale)
        into = b["G"]
        for k in (2, 1, 0):
            b["dW"].append(dg.weight_grad(s["H"][k], into))
            if k == 0:
                break
            b["dH"].append(dg.backward_data(into, self.W[k]))
            b["norm"].append(dg.group_norm_backward(s["P"][k - 1], b["dH"][-1], s["stats"][k - 1], self.dptr, **self.norm(k - 1)))
            into = dg.spmm(self.plan, b["norm"][-1].X, out_bf16=True)        # A is its own transpose
            b["dT"].append(into)
        return b

    def parameters(self):
        return [*self.W, *self.vec]

    @staticmethod
    def gradients(b):
        return [b["dW"][2], b["dW"][1], b["dW"][0], b["norm"][1].weight, b["norm"][1].bias, b["norm"][0].weight, b["norm"][0].bias]


@pytest.fixture(scope="module")
def batch(dg, device):
    return Batch(dg, device)


def check_spmm(batch, X, Y, what):
    want, B = oracle.spmm(batch.g, X.float().cpu().numpy())
    near(Y, want, 1e-5 * B, what)


def check_norms(batch, s):
    for k in range(2):
        p = batch.norm(k)
        Y, bound, st, rows = groupref.forward(host(s["P"][k]), batch.ptr, G, host(p["weight"]), host(p["bias"]), p["act"], EPS)
        near(s["H"][k + 1], Y, bound, f"norm {k}")
        assert (s["H"][k + 1][~rows] == 0).all()


def test_training_steps(dg, batch):
    s = batch.forward(dg.update)
    b = batch.backward(s)
    torch.cuda.synchronize()
    check_norms(batch, s)
    for k in range(2):
        product(s["T"][k], s["H"][k], batch.W[k], f"update {k}")
        check_spmm(batch, s["T"][k], s["P"][k], f"aggregation {k}")
    into = b["G"]
    for j, k in enumerate((2, 1)):
        product(b["dW"][j], s["H"][k].t().contiguous(), into, f"weight gradient {k}")
        product(b["dH"][j], into, batch.W[k].t().contiguous(), f"gradient's update {k}")
        p = batch.norm(k - 1)
        want = groupref.backward(host(s["P"][k - 1]), host(b["dH"][j]), batch.ptr, G, host(p["weight"]), host(p["bias"]), p["act"], EPS)
        for got, w, name in zip(b["norm"][j], want, ("X", "weight", "bias")):
            near(got, *w, f"d{name} of norm {k - 1}")
        check_spmm(batch, b["norm"][j].X, b["dT"][j], f"gradient's aggregation {k}")
        into = b["dT"][j]
    product(b["dW"][2], batch.X.t().contiguous(), into, "weight gradient 0")
    # the clipped step over all parameters, out of place and then in place
    grads, params = batch.gradients(b), batch.parameters()
    norm = math.sqrt(sum(float(t.double().square().sum()) for t in grads))
    most = 0.5 * norm
    new, got = dg.clipped_sgd(params, grads, 0.1, most, out=[torch.empty_like(t) for t in params])
    assert abs(got.item() - norm) <= 2.0 ** -24 * 1.001 * norm
    f = most / (norm + 1e-6)
    for t, w, g in zip(new, params, grads):
        want = host(w) - 0.1 * f * host(g)
        near(t, want, 1e-30, "step")
    clipped, _ = dg.clip_grads([t.clone() for t in grads], most)
    assert abs(dg.grad_norm(clipped).item() - most) <= 1e-5 * most
    # the same step again gives the same bits
    again = batch.gradients(batch.backward(batch.forward(dg.update)))
    assert all(torch.equal(x, y) for x, y in zip(again, grads))


def test_a_captured_training_step(dg, batch):
    """Forward, backward and the clipped step in one graph, replayed with other features and other graphs in the batch."""
    fresh = [t.clone() for t in batch.parameters()]
    out = [torch.empty_like(t) for t in fresh]

    def step():
        b = batch.backward(batch.forward(dg.update))
        _, norm = dg.clipped_sgd(batch.parameters(), batch.gradients(b), 0.1, 0.05, out=out)
        return b["loss"][:1], norm

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, norm = step()
    keep_x, keep_p = batch.X.clone(), batch.dptr.clone()
    try:
        for k in range(3):
            batch.X.normal_()
            batch.dptr.copy_(torch.from_numpy(np.sort(np.r_[0, np.random.default_rng(k).integers(0, batch.n, batch.ptr.size - 2), batch.n - k]).astype(np.int32)))
            want_loss, want_norm = step()
            want = [t.clone() for t in out]
            for t in out:
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(loss, want_loss) and torch.equal(norm, want_norm) and all(torch.equal(x, y) for x, y in zip(out, want))
    finally:
        batch.X.copy_(keep_x)
        batch.dptr.copy_(keep_p)


def four_bits(Q, s):
    t = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    t = np.concatenate([t, -t])
    q = Q.cpu().numpy()
    return t[np.stack([q & 15, q >> 4], 2).reshape(q.shape[0], -1)] * np.repeat(np.ldexp(1.0, s.cpu().numpy().astype(int) - 127), 32, 1)


def test_serving_in_4_bits(dg, batch):
    kept = {W.data_ptr(): dg.quantize_weight_mxfp4(W) for W in batch.W}      # weights are laid out once

    def update(X, W):
        q, sx = dg.quantize_mxfp4(X)
        wq, sw = kept[W.data_ptr()]
        T = dg.update_mxfp4(q, sx, wq, sw)
        a, w = four_bits(q, sx), four_bits(wq, sw)
        near(T, a @ w.T, 2 * 2.0 ** -24 * (a.shape[1] + 16) * (np.abs(a) @ np.abs(w).T), "4-bit update")
        one = dg.update_mxfp4(q[7:8].contiguous(), sx[7:8].contiguous(), wq, sw)      # a node by itself
        near(one, (a @ w.T)[7:8], 2 * 2.0 ** -24 * (a.shape[1] + 16) * (np.abs(a) @ np.abs(w).T)[7:8], "4-bit update of one node")
        return T

    s = batch.forward(update)
    torch.cuda.synchronize()
    check_norms(batch, s)
    for k in range(2):
        check_spmm(batch, s["T"][k], s["P"][k], f"aggregation {k}")
    # features kept in 4 bits are aggregated as the values they stand for
    q, sx = dg.quantize_mxfp4(batch.X)
    kept_x = dg.dequantize_mxfp4(q, sx, F_IN)
    assert np.array_equal(host(kept_x), four_bits(q, sx)[:, :F_IN])
    check_spmm(batch, kept_x, dg.spmm(batch.plan, kept_x), "aggregation of kept features")


def test_threads_on_streams_of_their_own(dg, batch, device):
    """Calls of ten host threads at once: every one has the bits of a call by itself."""
    s = batch.forward(dg.update)
    b = batch.backward(s)
    grads, params = batch.gradients(b), batch.parameters()
    W4 = dg.quantize_weight_mxfp4(batch.W[1])
    works = [lambda: dg.group_norm(s["P"][0], batch.dptr, **batch.norm(0)),
             lambda: tuple(dg.group_norm_backward(s["P"][1], b["dH"][0], s["stats"][1], batch.dptr, **batch.norm(1))),
             lambda: (dg.grad_norm(grads),),
             lambda: tuple(dg.clipped_sgd(params, grads, 0.1, 0.1, out=[torch.empty_like(t) for t in params])[0]),
             lambda: (dg.update_mxfp4(*dg.quantize_mxfp4(s["H"][1]), *W4),)]
    wants = [f() for f in works]
    torch.cuda.synchronize()

    def run(k):
        stream = torch.cuda.Stream(device)
        done = 0
        with torch.cuda.stream(stream):
            for _ in range(20):
                got = works[k]()
                assert len(got) == len(wants[k]) and all(torch.equal(x, y) for x, y in zip(got, wants[k])), k
                done += 1
            stream.synchronize()
        return done

    with ThreadPoolExecutor(10) as pool:
        for f in [pool.submit(run, k % 5) for k in range(10)]:
            assert f.result(timeout=60) == 20
