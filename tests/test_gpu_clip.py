"""The norm of many gradients, clipping and the clipped step on the GPU, against float64.

Tolerances, u = 2^-24: squares are exact in float64 and their sums off by less than 2^-40, so that the norm is a float32's
rounding off, u of itself; a result is formed in float64 (f to 2^-40) and rounded once, u of itself (bfloat16: once more,
2^-8 of itself), or half of the smallest float32 step."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = 2.0 ** -149


@pytest.fixture(scope="module")
def dg(device):
    import paper_2609_01983_amd as dg
    return dg


def make(device, sizes, bf16=(), size=0.1, seed=0):
    g = torch.Generator(device=device).manual_seed(seed + len(sizes))
    out = []
    for i, s in enumerate(sizes):
        t = torch.randn(s, device=device, generator=g) * size
        out.append(t.to(torch.bfloat16) if i in bf16 else t)
    return out


def exact_norm(grads):
    return math.sqrt(math.fsum(float(t.double().square().sum()) for t in grads))


def factor(norm, max_norm, eps):
    return 1.0 if norm + eps <= max_norm else max_norm / (norm + eps)


def near(got, want, what):
    bound = (1 + 2.0 ** -15) * U * want.abs() + TINY
    if got.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * want.abs() + 2.0 ** -134
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} outside"


def check(dg, grads, weights, max_norm, eps=1e-6, lr=0.3):
    norm = exact_norm(grads)
    for got in (dg.grad_norm(grads), dg.clip_grads(grads, max_norm, eps=eps, out=[torch.empty_like(t) for t in grads])[1]):
        if norm < 3.4e38:
            assert abs(got.item() - norm) <= (1 + 2.0 ** -15) * U * norm + TINY
        else:                                            # past float32's range; f is formed from the float64 norm
            assert got.item() == math.inf
    f = factor(norm, max_norm, eps)
    out, _ = dg.clip_grads(grads, max_norm, eps=eps, out=[torch.empty_like(t) for t in grads])
    for i, (o, t) in enumerate(zip(out, grads)):
        near(o, f * t.double(), f"clipped {i}")
    keep = [w.clone() for w in weights]
    new, n2 = dg.clipped_sgd(weights, grads, lr, max_norm, eps=eps, out=[torch.empty_like(w) for w in weights])
    for i, (o, w, t) in enumerate(zip(new, weights, grads)):
        near(o, w.double() - lr * f * t.double(), f"step {i}")
        assert torch.equal(w, keep[i])
    # in place: the same bits
    same, n3 = dg.clipped_sgd(keep, grads, lr, max_norm, eps=eps)
    assert same is keep and all(torch.equal(a, b) for a, b in zip(keep, new)) and torch.equal(n2, n3)
    mine = [t.clone() for t in grads]
    dg.clip_grads(mine, max_norm, eps=eps)
    assert all(torch.equal(a, b) for a, b in zip(mine, out))


@pytest.mark.parametrize("sizes", [[(1,)], [(0,)], [(0,), (3,), (0,)], [(2, 2)], [(5,), (4, 7), (1,), (33, 3)], [(8191,), (8192,), (8193,)],
                                   [(256, 128), (128, 64)], [(1 << 20,), (3,), (300, 700)], [(65, 129)] * 40])
@pytest.mark.parametrize("max_norm", [0.01, 1.0, 1e9])
def test_sizes(dg, device, sizes, max_norm):
    check(dg, make(device, sizes), make(device, sizes, seed=9), max_norm)
    check(dg, make(device, sizes, bf16=range(0, len(sizes), 2)), make(device, sizes, seed=9), max_norm)


@pytest.mark.parametrize("tensors", [88, 89, 160, 161, 999])
def test_many_tensors(dg, device, tensors):
    """More than one launch's arguments hold."""
    sizes = [(1 + 37 * i % 311,) for i in range(tensors)]
    sizes[tensors // 2] = (50000,)
    check(dg, make(device, sizes, bf16=range(1, tensors, 3)), make(device, sizes, seed=1), 0.5)


def test_large(dg, device):
    sizes = [(4096, 4096), (17,), (5000, 5001)]
    check(dg, make(device, sizes, bf16=(2,)), make(device, sizes, seed=3), 2.0)


def test_more_than_2_to_the_31_elements(dg, device):
    n = (1 << 31) + 12345
    g = torch.full((n,), 0.5, device=device, dtype=torch.bfloat16)
    g[-1] = 4096.0
    norm = math.sqrt(0.25 * (n - 1) + 4096.0 ** 2)
    out, got = dg.clip_grads([g], 1.0)
    assert out[0] is g and abs(got.item() - norm) <= 1.001 * U * norm
    f = 1.0 / (norm + 1e-6)
    ends = g[[0, 1 << 30, n - 2, n - 1]].double().cpu()
    want = torch.tensor([0.5, 0.5, 0.5, 4096.0], dtype=torch.float64) * f
    assert ((ends - want).abs() <= 2.0 ** -8 * 1.001 * want).all()


def test_extremes(dg, device):
    """Squares that are no float32 numbers, subnormal gradients, and f below float32's range."""
    big = [torch.full((1000,), 3e38, device=device), torch.randn(77, device=device)]
    check(dg, big, [torch.zeros(1000, device=device), torch.ones(77, device=device)], 1.0)
    small = [torch.full((3000,), 1e-41, device=device), torch.full((5,), 1e-30, device=device)]
    check(dg, small, [torch.zeros(3000, device=device), torch.ones(5, device=device)], 1e-33, eps=0.0)
    zero = [torch.zeros(50, device=device)]
    out, norm = dg.clip_grads(zero, 0.0, eps=0.0)
    assert norm.item() == 0 and (out[0] == 0).all()
    some = make(device, [(300,)])
    out, norm = dg.clip_grads(some, 0.0, out=[torch.empty_like(some[0])])
    assert (out[0] == 0).all() and norm.item() > 0
    out, norm = dg.clip_grads(some, math.inf, out=[torch.empty_like(some[0])])
    assert torch.equal(out[0], some[0])


def test_not_finite(dg, device):
    grads = make(device, [(500,), (70, 3)])
    grads[1][5, 1] = float("inf")
    out, norm = dg.clip_grads(grads, 1.0, out=[torch.empty_like(t) for t in grads])
    assert norm.item() == math.inf and (out[0] == 0).all() and torch.isnan(out[1][5, 1])
    grads[0][3] = float("nan")
    out, norm = dg.clip_grads(grads, 1.0, out=[torch.empty_like(t) for t in grads])
    assert all(torch.isnan(t).all() for t in [norm, *out])
    assert torch.isnan(dg.grad_norm(grads)).all()


def test_odd_places(dg, device):
    """Tensors side by side in one piece of memory at any element; nothing between them is written."""
    for t in (torch.float32, torch.bfloat16):
        buf = torch.randn(40000, device=device).to(t)
        cuts = [(1, 20), (23, 9001), (9003, 9004), (9005, 30011), (30014, 39997)]
        grads = [buf[a:b] for a, b in cuts]
        weights = make(device, [(b - a,) for a, b in cuts])
        check(dg, grads, weights, 0.7)
        out = torch.full((40000,), 5.0, device=device, dtype=t)
        dg.clip_grads(grads, 0.7, out=[out[a:b] for a, b in cuts])
        rest = torch.ones(40000, dtype=torch.bool, device=device)
        for a, b in cuts:
            rest[a:b] = False
        assert (out[rest] == 5).all() and not (out[~rest] == 5).all()


def test_the_same_gradient_twice(dg, device):
    g = make(device, [(999,)])[0]
    assert abs(dg.grad_norm([g, g]).item() - math.sqrt(2) * exact_norm([g])) <= 2 * U * math.sqrt(2) * exact_norm([g])
    w = make(device, [(999,), (999,)], seed=5)
    new, _ = dg.clipped_sgd(w, [g, g], 0.1, 1e9, out=[torch.empty_like(x) for x in w])
    for a, b in zip(new, w):
        near(a, b.double() - 0.1 * g.double(), "step")
    with pytest.raises(dg.DualGCNError) as e:            # in place it would be scaled twice
        dg.clip_grads([g, g], 1.0)
    assert e.value.status == dg.ERR_INVALID_ARG


def test_results_do_not_depend_on_timing(dg, device):
    grads = make(device, [(3000, 700), (123457,), (5,)])
    want = dg.clip_grads(grads, 1.0, out=[torch.empty_like(t) for t in grads])
    for _ in range(5):
        got = dg.clip_grads(grads, 1.0, out=[torch.empty_like(t) for t in grads])
        assert torch.equal(got[1], want[1]) and all(torch.equal(a, b) for a, b in zip(got[0], want[0]))


def test_streams_and_graphs(dg, device):
    for sizes in ([(64, 32), (5,)], [(300, 500)] * 170):
        grads, weights = make(device, sizes), make(device, sizes, seed=2)
        out = [torch.empty_like(t) for t in weights]

        def call(stream=None):
            _, norm = dg.clipped_sgd(weights, grads, 0.1, 1.0, out=out, stream=stream)
            return norm

        norm = call()
        want = [t.clone() for t in out]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        n2 = call(side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(n2, norm) and all(torch.equal(a, b) for a, b in zip(out, want))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cap = call()
        for k in range(3):
            for t in grads:
                t.normal_(std=0.01 * (k + 1))
            norm = call()
            want = [t.clone() for t in out]
            for t in out:
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(cap, norm) and all(torch.equal(a, b) for a, b in zip(out, want))


def test_lists_in_place(dg, device):
    """The same list, or another with the same tensors, is in place; weights cannot go to the gradients' places."""
    g, w = make(device, [(10,), (4, 5), (0,)]), make(device, [(10,), (4, 5), (0,)])
    g[1] = g[1].to(torch.bfloat16)
    want, norm = dg.clip_grads(g, 0.5, out=[torch.empty_like(t) for t in g])
    new, _ = dg.clipped_sgd(w, g, 0.1, 0.5, out=[torch.empty_like(t) for t in w])
    for same in (lambda v: v, list, tuple):
        a, b, c = [t.clone() for t in g], [t.clone() for t in w], [t.clone() for t in g]
        out, n = dg.clip_grads(a, 0.5, out=same(a))
        assert torch.equal(n, norm) and all(torch.equal(x, y) for x, y in zip(out, want)) and out[0] is a[0]
        out, n = dg.clipped_sgd(tuple(b), tuple(c), 0.1, 0.5, out=same(b))
        assert torch.equal(n, norm) and all(torch.equal(x, y) for x, y in zip(out, new)) and out[0] is b[0]
    c = [t.float() for t in g]
    with pytest.raises(dg.DualGCNError):
        dg.clipped_sgd(w, c, 0.1, 1.0, out=c)
    with pytest.raises(TypeError):
        dg.clip_grads(c, 1.0, out=[t.cpu() for t in c])


def test_refusals(dg, device):
    g, w = make(device, [(10,), (4, 5)]), make(device, [(10,), (4, 5)])
    for bad in (lambda: dg.grad_norm([]), lambda: dg.clipped_sgd(w[:1], g, 0.1, 1.0), lambda: dg.clip_grads(g, 1.0, out=g[:1]),
                lambda: dg.clipped_sgd([w[0], w[1].t().contiguous()], g, 0.1, 1.0), lambda: dg.grad_norm([g[1].t()])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: dg.grad_norm([g[0].double()]), lambda: dg.grad_norm([g[0].cpu()]), lambda: dg.grad_norm([3.0]),
                lambda: dg.clipped_sgd([t.to(torch.bfloat16) for t in w], g, 0.1, 1.0)):
        with pytest.raises(TypeError):
            bad()
    flat = torch.zeros(100, device=device)
    for bad in (lambda: dg.clip_grads(g, -1.0), lambda: dg.clip_grads(g, math.nan), lambda: dg.clip_grads(g, 1.0, eps=-1.0),
                lambda: dg.clipped_sgd(w, g, math.inf, 1.0), lambda: dg.clip_grads([flat[:50]], 1.0, out=[flat[10:60]]),
                lambda: dg.clip_grads([flat[:50], flat[50:]], 1.0, out=[flat[50:], flat[:50]]),
                lambda: dg.clipped_sgd([flat[:10], flat[5:15]], [g[0], g[0]], 0.1, 1.0),
                lambda: dg.grad_norm(g, workspace=torch.empty(100, dtype=torch.uint8, device=device))):
        with pytest.raises(dg.DualGCNError) as e:
            bad()
        assert e.value.status == dg.ERR_INVALID_ARG
