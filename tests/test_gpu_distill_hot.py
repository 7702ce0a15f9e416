"""The distillation loss at high temperatures, where the divergence falls as 1 / T^2 and the loss,
T^2 of it, does not: against float64, relative to the loss itself.

Bound, v = 2^-53: a row's soft loss is T^2 times (sum p (z_t - z_y) + log S_y - log S_t), in float64.  The sums of
exponentials are of terms off by 4 v, in chains of C / 16 at most here and 10 joins; a logarithm of them is at
most log C + 1 in size.  Altogether v (16 + C / 16 + 2 log C) T^2 a row on each side (numpy's sums are pairwise: less).
The result is rounded to float32 once and its scale holds T^2 soft_scale to float64: u = 2^-24, and 2 u where soft and hard are added."""
import numpy as np
import pytest
import torch

from test_gpu_distill import CLASSES, INF, _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dg(device):
    import paper_2609_01983_amd as dg
    return dg


def _soft(Y, ids, teacher, T):
    """T^2 sum p (log p - log Q[id]) over the rows, in float64."""
    total = 0.0
    for v in range(len(Y)):
        ok = (ids[v] >= 0) & (ids[v] < Y.shape[1]) & ~(teacher[v] == -np.inf)
        if not ok.any():
            continue
        t = (teacher[v][ok] - teacher[v][ok].max()) / T
        y = (Y[v] - Y[v].max()) / T
        p = np.exp(t) / np.exp(t).sum()
        total += (p * (t - y[ids[v][ok]])).sum() + np.log(np.exp(y).sum()) - np.log(np.exp(t).sum())
    return T * T * total


# every class kept: only then the divergence is small; few and many rows, short and long
@pytest.mark.parametrize("n,C", [(1, 2), (300, 3), (40, 47), (5000, 64), (77, 128), (33, 700), (9, 1025), (5, 4096)])
@pytest.mark.parametrize("T", [8.5, 100.0, 1000.0, 16384.0])
@pytest.mark.parametrize("y,t", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16),
                                 (torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)])
def test_every_class_kept(dg, device, n, C, T, y, t):
    rng = np.random.default_rng(n + C)
    make = lambda d: torch.from_numpy((2 * rng.standard_normal((n, C))).astype(np.float32)).to(d).to(device)  # noqa: E731
    Y, teacher = make(y), make(t)
    ids = torch.from_numpy(np.argsort(rng.random((n, C)), axis=1).astype(np.int32)).to(device)
    scale = 1.0 / 128
    _, loss = dg.distill_xent(Y, ids, teacher, temperature=T, soft_scale=scale)
    want = scale * _soft(Y.double().cpu().numpy(), ids.cpu().numpy(), teacher.double().cpu().numpy(), T)
    bound = 2.0 ** -24 * abs(want) + 2 * 2.0 ** -53 * (16 + C / 16 + 2 * np.log(C)) * T * T * scale * n
    lo = loss.double().cpu().numpy()
    assert abs(lo[1] - want) <= bound and abs(lo[0] - want) <= 3 * bound and lo[2] == 0.0, (lo, want, bound)
    assert want > 0


@pytest.mark.parametrize("C", CLASSES)
def test_every_width(dg, device, C):
    """Loss and gradient past the border as on this side of it, labels, missing entries and all."""
    for n, K in ((1, 1), (6, 5), (35, 40)):
        a = _inputs(device, n, C, K, seed=n)
        _check(dg, *a, T=20.0)
        b = dg.distill_xent(*a, temperature=20.0, soft_scale=0.3, hard_scale=0.2)
        c = dg.distill_xent(*a, temperature=20.0, soft_scale=0.3, hard_scale=0.2)
        assert torch.equal(b[0], c[0]) and torch.equal(b[1], c[1])


@pytest.mark.parametrize("C", [2, 40, 130, 700, 3000, 50000])
def test_logits_that_are_not_finite(dg, device, C):
    Y, ids, teacher, labels = _inputs(device, 24, C, 6, missing=0.0)
    ids[:] = torch.arange(6, device=device) % C
    labels[:] = -1
    lowest = torch.finfo(torch.float32).min
    Y[1, C // 2:] = -INF
    Y[1, 0] = 0.0
    ids[1] = -1
    ids[1, 0] = 0
    Y[3] = lowest
    Y[4] = -INF
    Y[6, 0] = float("nan")
    Y[7, C - 1] = INF
    Y[8, 0] = -INF
    teacher[9] = -INF
    Y[9] = float("nan")
    teacher[11, 0] = -INF
    teacher[12, 0] = float("nan")
    teacher[13, 1] = INF
    teacher[14] = lowest
    for rows in ([0, 1, 3, 9, 11, 14, 16, 17], [4], [6], [7], [8], [12], [13]):
        pick = lambda x: x[rows].contiguous()  # noqa: E731
        _check(dg, pick(Y), pick(ids), pick(teacher), pick(labels), T=10.0)


def test_streams_and_graphs(dg, device):
    for n, C in ((37, 45), (19, 700), (5, 30001)):
        Y, ids, teacher, labels = _inputs(device, n, C, 6)
        call = lambda X, **k: dg.distill_xent(X, ids, teacher, labels, temperature=30.0, soft_scale=0.1, hard_scale=0.1, **k)  # noqa: E731
        want = call(Y)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = call(Y, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        torch.cuda.synchronize()
        X = Y.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cap = call(X)
        for k in range(3):
            X.copy_(Y * (1 + k))
            eager = call(X)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(cap[0], eager[0]) and torch.equal(cap[1], eager[1])
    with pytest.raises(dg.DualGCNError) as e:
        call(Y, workspace=torch.empty(dg.distill_workspace_bytes(5, 30001, 6) - 256, dtype=torch.uint8, device=device))
    assert e.value.status == dg.ERR_INVALID_ARG
