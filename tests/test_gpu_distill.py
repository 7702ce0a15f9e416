"""The distillation loss and its gradient on the GPU against float64 (distillref.py, whose bounds
are derived there): classes over every width class and its borders, few and many rows, types,
rows without a teacher or label, ids given twice, infinities and NaN; gradients against
differences; streams, graphs, refusals."""
import numpy as np
import pytest
import torch

import distillref as ref

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.fixture(scope="module")
def dg(device):
    import paper_2609_01983_amd as dg
    return dg


def _inputs(device, n, C, K, seed=0, y="f32", t="f32", labels=True, missing=0.2, spread=3.0):
    rng = np.random.default_rng(seed + 7919 * n + 104729 * C + K)
    types = {"f32": torch.float32, "bf16": torch.bfloat16}
    Y = torch.from_numpy((rng.standard_normal((n, C)) * spread).astype(np.float32)).to(types[y])
    teacher = torch.from_numpy((rng.standard_normal((n, K)) * 2 + 4).astype(np.float32)).to(types[t])
    ids = np.empty((n, K), dtype=np.int32)
    for v in range(n):                                   # distinct where there are classes enough
        ids[v] = rng.choice(C, K, replace=K > C)
    ids[rng.random((n, K)) < missing] = -1
    ids[rng.random((n, K)) < missing / 4] = C + 5
    ids[::5] = -1                                        # rows without a teacher
    lab = rng.integers(0, C, n).astype(np.int32)
    lab[rng.random(n) < 0.5] = -1
    lab[::7] = C
    lab = torch.from_numpy(lab) if labels else None
    return (Y.to(device), torch.from_numpy(ids).to(device), teacher.to(device),
            lab.to(device) if labels else None)


def _check(dg, Y, ids, teacher, labels, T=1.0, soft=0.3, hard=0.2, grad_bf16=False, **more):
    G, loss = dg.distill_xent(Y, ids, teacher, labels, temperature=T, soft_scale=soft, hard_scale=hard,
                              grad_bf16=grad_bf16, **more)
    h = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
    # the scales as the library holds them
    soft, hard = float(np.float32(soft)), float(np.float32(hard))
    wG, wl, bG, bl = ref.distill(Y.double().cpu().numpy(), h(ids), teacher.double().cpu().numpy(), h(labels), T, soft, hard)
    g = G.double().cpu().numpy()
    bound = bG + (ref.BF16 * (np.abs(wG) + bG) if grad_bf16 else 2 * ref.U * np.abs(wG))
    fine = np.isfinite(wG)
    assert np.array_equal(fine, np.isfinite(g)), "non-finite gradients elsewhere"
    bad = fine & ~(np.abs(np.where(fine, g - wG, 0.0)) <= np.where(fine, bound, 0.0))
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"G: {bad.sum()} outside; at {i} got {g[i]!r} want {wG[i]!r} bound {bound[i]!r}")
    lo = loss.double().cpu().numpy()
    for k in range(3):
        if np.isfinite(wl[k]):
            assert abs(lo[k] - wl[k]) <= bl[k], (k, lo, wl, bl)
        else:
            assert np.isnan(lo[k]) if np.isnan(wl[k]) else lo[k] == wl[k], (k, lo, wl)
    return G, loss


CLASSES = [1, 2, 3, 4, 5, 31, 32, 33, 47, 64, 65, 128, 129, 255, 256, 257, 512, 513, 1000, 1024, 1025, 2048, 2049, 4096,
           4097, 8191, 8192, 8193, 16384, 16385, 40003]


@pytest.mark.parametrize("C", CLASSES)
@pytest.mark.parametrize("T", [1.0, 2.5])
def test_every_width(dg, device, C, T):
    for n, K in ((1, 1), (6, 5), (35, 40)):
        _check(dg, *_inputs(device, n, C, K, seed=n), T=T)


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("labels", [True, False])
def test_types(dg, device, y, t, labels):
    for C in (3, 47, 600, 3000, 20001):
        for half in (False, True):
            _check(dg, *_inputs(device, 23, C, 9, y=y, t=t, labels=labels), T=0.5, grad_bf16=half)


@pytest.mark.parametrize("C,K", [(10, 300), (100, 129), (700, 700), (5000, 1100), (30000, 4096)])
def test_many_entries(dg, device, C, K):
    """More entries than a row's threads hold, and (K > C) ids given more than twice."""
    _check(dg, *_inputs(device, 11, C, K), T=2.0)


@pytest.mark.parametrize("C", [5, 64, 300, 2000, 9000, 50000])
def test_an_id_given_twice(dg, device, C):
    Y, ids, teacher, labels = _inputs(device, 16, C, 12, missing=0.0)
    ids[1] = ids[1, 0]                                   # all entries the same class
    ids[2, 1] = ids[2, 0]
    ids[3, 6:] = ids[3, :6]
    a = _check(dg, Y, ids, teacher, labels, T=3.0)
    b = dg.distill_xent(Y, ids, teacher, labels, temperature=3.0, soft_scale=0.3, hard_scale=0.2)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("n,C", [(4099, 64), (20001, 3), (3001, 128), (700, 9001), (257, 20000), (3, 200000), (1, 1000003)])
def test_many_rows_and_long_ones(dg, device, n, C):
    """Rows beyond one step of the grid, and long rows that workgroups share; the same bits twice."""
    args = _inputs(device, n, C, 8) if n < 5000 else _inputs(device, n, C, 2)
    a = _check(dg, *args, T=2.0, soft=1.0 / n, hard=1.0 / n)
    b = dg.distill_xent(*args, temperature=2.0, soft_scale=1.0 / n, hard_scale=1.0 / n)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", [(1, 32768), (128, 32768), (128, 32769), (129, 32769), (130, 40000), (127, 40000)])
def test_around_the_longest_held_and_the_last_split_rows(dg, device, n, C, y):
    _check(dg, *_inputs(device, n, C, 8, y=y), T=2.0, soft=1.0 / n, hard=1.0 / n)


@pytest.mark.parametrize("C", [2, 40, 130, 700, 3000, 12000, 50000])
def test_masked_infinite_and_nan_logits(dg, device, C):
    Y, ids, teacher, labels = _inputs(device, 24, C, 6, missing=0.0)
    ids[:] = torch.arange(6, device=device) % C
    labels[:] = -1
    lowest = torch.finfo(torch.float32).min
    Y[1, C // 2:] = -INF                                 # masked classes
    Y[1, 0] = 0.0
    ids[1] = -1
    ids[1, 0] = 0
    Y[2, 1:] = lowest                                    # masks of the type's lowest value
    Y[3] = lowest                                        # every class masked by it: uniform
    Y[4] = -INF                                          # nothing left: NaN
    Y[6, 0] = float("nan")
    Y[7, C - 1] = INF
    Y[8, 0] = -INF                                       # the teacher takes a masked class: infinite loss
    teacher[9] = -INF                                    # no entry, no label: zeros
    Y[9] = float("nan")
    teacher[11, 0] = -INF                                # one entry fewer
    teacher[12, 0] = float("nan")
    teacher[13, 1] = INF
    teacher[14] = lowest
    labels[16] = C - 1
    ids[16] = -1
    Y[17] = Y[17] * 1e4                                  # one class has it all
    teacher[18] = teacher[18] * 1e4
    for rows in ([0, 1, 2, 3, 9, 11, 14, 16, 17, 18], [4], [6], [7], [8], [12], [13]):
        for T in (1.0, 2.0):
            pick = lambda t: t[rows].contiguous()  # noqa: E731
            G, loss = _check(dg, pick(Y), pick(ids), pick(teacher), pick(labels), T=T)
    # a bad row leaves the others as they are
    G, _ = dg.distill_xent(Y, ids, teacher, labels, temperature=2.0, soft_scale=0.3, hard_scale=0.2)
    good = [0, 1, 2, 3, 9, 11, 14, 16, 17, 18, 19, 21, 22]
    alone, _ = dg.distill_xent(Y[good].contiguous(), ids[good].contiguous(), teacher[good].contiguous(),
                               labels[good].contiguous(), temperature=2.0, soft_scale=0.3, hard_scale=0.2)
    assert torch.allclose(G[good], alone, rtol=1e-5, atol=1e-9)
    assert torch.equal(G[9], torch.zeros_like(G[9]))


@pytest.mark.parametrize("n,C", [(300000, 5), (70000, 300), (33000, 600), (9000, 1100), (9000, 5001), (300, 20001), (8300, 33000)])
def test_rows_beside_a_teacher_that_is_not_finite(dg, device, n, C):
    """Rows whose teacher has a +infinity or a NaN leave the rows behind them as they were, and have NaN at
    the classes of their entries only (an entry of -infinity is none)."""
    g = torch.Generator(device=device).manual_seed(C)
    Y = torch.randn(n, C, device=device, generator=g)
    K = 5
    start = torch.randint(0, C, (n, 1), device=device, generator=g)
    ids = ((start + torch.arange(K, device=device) * (C // K)) % C).int()     # distinct
    teacher = torch.randn(n, K, device=device, generator=g)
    want, _ = dg.distill_xent(Y, ids, teacher, temperature=2.0, soft_scale=0.1)
    bad = torch.arange(n, device=device) % 7 == 3
    poisoned = teacher.clone()
    poisoned[bad, 1] = float("inf")
    poisoned[3, 1] = float("nan")
    poisoned[bad, 2] = -float("inf")
    got, loss = dg.distill_xent(Y, ids, poisoned, temperature=2.0, soft_scale=0.1)
    assert torch.equal(got[~bad], want[~bad])
    nan = torch.zeros(int(bad.sum()), C, dtype=torch.bool, device=device)
    nan.scatter_(1, ids[bad][:, [0, 1, 3, 4]].long(), True)
    assert torch.equal(got[bad].isnan(), nan) and loss[0].isnan()


def test_gradient_against_differences(dg, device):
    """The loss in float64, differenced along random directions: the step 1e-5 leaves 1e-10 of the
    third derivatives and 1e-11 / 1e-5 of rounding, far below the allowance."""
    Y, ids, teacher, labels = _inputs(device, 9, 21, 5)
    G, _ = dg.distill_xent(Y, ids, teacher, labels, temperature=2.0, soft_scale=0.3, hard_scale=0.2)
    G = G.double().cpu().numpy()
    y, i, t, lab = Y.double().cpu().numpy(), ids.cpu().numpy(), teacher.double().cpu().numpy(), labels.cpu().numpy()
    rng = np.random.default_rng(0)
    for _ in range(4):
        v = rng.standard_normal(y.shape)
        up, down = (ref.distill(y + h * v, i, t, lab, 2.0, 0.3, 0.2)[1][0] for h in (1e-5, -1e-5))
        assert abs((G * v).sum() - (up - down) / 2e-5) <= 1e-5 * np.abs(G * v).sum() + 1e-6


def test_agrees_with_softmax_xent(dg, device):
    """Without entries the loss is dualgcn_softmax_xent's; a teacher sure of one class is a label."""
    Y, ids, teacher, labels = _inputs(device, 500, 47, 4)
    none = torch.full_like(ids, -1)
    scale = 1.0 / 500
    G, loss = dg.distill_xent(Y, none, teacher, labels, soft_scale=scale, hard_scale=scale)
    G1, loss1 = dg.softmax_xent(Y, labels, scale)
    assert torch.allclose(G, G1, rtol=1e-5, atol=1e-5 * scale) and abs(loss[0].item() - loss1[0].item()) <= 1e-5
    sure = labels[:, None].contiguous()
    G, loss = dg.distill_xent(Y, sure, torch.zeros(500, 1, device=device), soft_scale=scale)
    assert torch.allclose(G, G1, rtol=1e-5, atol=1e-5 * scale) and abs(loss[1].item() - loss1[0].item()) <= 1e-5


def test_default_scales(dg, device):
    Y, ids, teacher, labels = _inputs(device, 60, 10, 3)
    taught = ((ids >= 0) & (ids < 10)).any(1).sum().item()
    labeled = ((labels >= 0) & (labels < 10)).sum().item()
    a = dg.distill_xent(Y, ids, teacher, labels)
    b = dg.distill_xent(Y, ids, teacher, labels, soft_scale=1.0 / taught, hard_scale=1.0 / labeled)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_default_scales_wait_for_the_stream(dg, device):
    Y, ids, teacher, labels = _inputs(device, 60, 10, 3)
    want = dg.distill_xent(Y, ids, teacher, labels)
    late, late_labels = torch.full_like(ids, -1), torch.full_like(labels, -1)
    busy = torch.eye(4096, device=device)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(20):
            busy = busy @ busy
        late.copy_(ids)
        late_labels.copy_(labels)
    got = dg.distill_xent(Y, late, teacher, late_labels, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_views_streams_and_graphs(dg, device):
    for n, C in ((37, 45), (19, 700), (5, 30001)):
        Y, ids, teacher, labels = _inputs(device, n, C, 6)
        want = dg.distill_xent(Y, ids, teacher, labels, temperature=2.0, soft_scale=0.1, hard_scale=0.1)
        flat = torch.empty(n * C + 5, device=device)
        V = flat[1:1 + n * C].view(n, C).copy_(Y)
        out = torch.full((n * C + 7,), 9.0, device=device)
        G, loss = dg.distill_xent(V, ids, teacher, labels, temperature=2.0, soft_scale=0.1, hard_scale=0.1,
                                  G=out[3:3 + n * C].view(n, C))
        assert torch.equal(G, want[0]) and torch.equal(loss, want[1])
        assert (out[:3] == 9).all() and (out[3 + n * C:] == 9).all()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = dg.distill_xent(Y, ids, teacher, labels, temperature=2.0, soft_scale=0.1, hard_scale=0.1, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        torch.cuda.synchronize()
        X = Y.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cap = dg.distill_xent(X, ids, teacher, labels, temperature=2.0, soft_scale=0.1, hard_scale=0.1)
        for k in range(3):
            X.copy_(Y * (1 + k))
            eager = dg.distill_xent(X, ids, teacher, labels, temperature=2.0, soft_scale=0.1, hard_scale=0.1)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(cap[0], eager[0]) and torch.equal(cap[1], eager[1])


def test_more_than_2_to_the_31_logits(dg, device):
    n, C = (1 << 17) + 1, 16500
    Y = torch.empty(n, C, device=device, dtype=torch.bfloat16)
    for a in range(0, n, 1 << 14):
        Y[a:a + (1 << 14)].normal_()
    ids = torch.zeros(n, 1, dtype=torch.int32, device=device)
    teacher = torch.zeros(n, 1, device=device)
    G, _ = dg.distill_xent(Y, ids, teacher, soft_scale=1.0, grad_bf16=True)
    rows = torch.tensor([0, n // 2, n - 2, n - 1], device=device)
    _check(dg, Y[rows].contiguous(), ids[:4], teacher[:4], None, soft=1.0, grad_bf16=True)
    want, _ = dg.distill_xent(Y[rows].repeat(200, 1), ids[:800], teacher[:800], soft_scale=1.0, grad_bf16=True)
    assert torch.equal(G[rows], want[:4])


def test_refusals(dg, device):
    Y, ids, teacher, labels = _inputs(device, 8, 20, 3)
    with pytest.raises(TypeError):
        dg.distill_xent(Y.cpu(), ids, teacher)
    with pytest.raises(TypeError):
        dg.distill_xent(Y, ids.long(), teacher)
    with pytest.raises(ValueError):
        dg.distill_xent(Y, ids[:4].contiguous(), teacher)
    with pytest.raises(ValueError):
        dg.distill_xent(Y, ids, teacher[:, :2].contiguous())
    with pytest.raises(ValueError):
        dg.distill_xent(Y.t(), ids, teacher)
    with pytest.raises(ValueError):
        dg.distill_xent(Y, ids, teacher, labels[:3].contiguous())
    for bad in (dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=INF), dict(temperature=float("nan")),
                dict(soft_scale=INF), dict(hard_scale=float("nan")), dict(G=Y)):
        with pytest.raises(dg.DualGCNError) as e:
            dg.distill_xent(Y, ids, teacher, labels, **dict(dict(soft_scale=1.0, hard_scale=1.0), **bad))
        assert e.value.status == dg.ERR_INVALID_ARG
    with pytest.raises(dg.DualGCNError) as e:
        dg.distill_xent(Y, ids, teacher, workspace=torch.empty(16, dtype=torch.uint8, device=device))
    assert e.value.status == dg.ERR_INVALID_ARG
    wide = torch.zeros(8, 4097, dtype=torch.int32, device=device)
    with pytest.raises(dg.DualGCNError) as e:
        dg.distill_xent(Y, wide, wide.float())
    assert e.value.status == dg.ERR_UNSUPPORTED
