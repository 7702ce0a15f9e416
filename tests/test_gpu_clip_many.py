"""Clipping and the clipped step over very many tensors on the GPU: results against float64, and a cost that goes with their number.

Tolerances as for few tensors: the norm's rounding to float32, 2^-24 of itself; a result formed in float64 and rounded
once, 2^-24 of itself."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def dg(device):
    import paper_2609_01983_amd as dg
    return dg


def make(device, tensors, each, seed=0):
    g = torch.Generator(device=device).manual_seed(seed)
    flat = torch.randn(tensors * each, device=device, generator=g) * 0.1
    return flat, list(flat.split(each))


def near(got, want):
    assert ((got.double() - want).abs() <= (1 + 2.0 ** -15) * U * want.abs() + 2.0 ** -149).all()


# partial sums of less than one, of four, of just over four and of many launches
@pytest.mark.parametrize("tensors,each", [(300, 8192 * 3), (640, 8192 * 13), (641, 8192 * 13), (1000, 100000), (9000, 5)])
def test_many_partial_sums(dg, device, tensors, each):
    flat, grads = make(device, tensors, each)
    wflat, weights = make(device, tensors, each, 1)
    norm = math.sqrt(float(flat.double().square().sum()))
    oflat = torch.empty_like(flat)
    for most in (1.0, 1e9):
        f = min(1.0, most / (norm + 1e-6))
        _, n1 = dg.clip_grads(grads, most, out=list(oflat.split(each)))
        near(oflat, f * flat.double())
        _, n2 = dg.clipped_sgd(weights, grads, 0.3, most, out=list(oflat.split(each)))
        near(oflat, wflat.double() - 0.3 * f * flat.double())
        n3 = dg.grad_norm(grads)
        assert abs(n1.item() - norm) <= (1 + 2.0 ** -15) * U * norm and torch.equal(n1, n2) and torch.equal(n1, n3)
    flat[-1] = float("inf")
    _, n1 = dg.clip_grads(grads, 1.0, out=list(oflat.split(each)))
    assert n1.item() == math.inf and (oflat[:-1] == 0).all() and torch.isnan(oflat[-1])


def test_the_cost_goes_with_the_number(dg, device):
    """2^17 small tensors, captured, so that only launches and kernels are timed: the step has the norm's launches and not quite twice as many of
    its own, of two operands and a result: some three times the norm's time.  (Where each of its workgroups
    summed all partial sums it was 9.6 times, and twice that for twice the tensors.)"""
    flat, grads = make(device, 1 << 17, 4)
    wflat, weights = make(device, 1 << 17, 4, 1)
    oflat = torch.empty_like(flat)
    out = list(oflat.split(4))
    calls = [lambda: dg.grad_norm(grads), lambda: dg.clipped_sgd(weights, grads, 0.3, 1.0, out=out)[1]]
    times = []
    for call in calls:
        want = call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            norm = call()
        took = []
        for _ in range(5):
            oflat.zero_()
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            graph.replay()
            end.record()
            end.synchronize()
            took.append(start.elapsed_time(end))
            assert torch.equal(norm, want)
        times.append(sorted(took)[2])
    exact = math.sqrt(float(flat.double().square().sum()))
    near(oflat, wflat.double() - 0.3 / (exact + 1e-6) * flat.double())
    assert times[1] <= 5 * times[0], times
