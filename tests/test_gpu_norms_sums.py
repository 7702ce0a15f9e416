"""The norms around a block over many rows: column sums of passes so long that they are done in parts,
rows over several steps of every shape, and outputs past 32 MiB with a block and every pair of types.

A column sum adds at most 128 rows in float32 one after another (a group of threads), then at most 31 groups, all else
in float64: 160 roundings, each of at most u = 2^-24 of the sum so far, which for terms of one sign
grows to the whole sum evenly: 80 u of the terms' magnitudes, and K_BACK u (normref.py) for the terms themselves."""
import numpy as np
import pytest
import torch

import normref as ref
from test_gpu_norms import _case, _check_backward, _check_forward

pytestmark = pytest.mark.gpu

SUM = ref.U * (80 + ref.K_BACK)


@pytest.fixture(scope="module")
def dg(device):
    import paper_2609_01983_amd as dg
    return dg


def test_a_long_column_of_equal_terms(dg, device):
    """67 million rows: a chain of float32 additions over all rows of a workgroup is off by far more."""
    n, F = (1 << 26) + 3, 4
    Rn = torch.arange(n * F, device=device, dtype=torch.int32).remainder_(97).float().view(n, F)
    dZ = torch.full((n, F), 0.1, device=device)
    zero, scale = torch.zeros(F, device=device), float(np.float32(0.3))
    got = dg.norm_residual_backward(Rn, Rn, dZ, dZ, post_bias=zero, pre_bias=zero, kind="layer", scale=scale)
    term = float(np.float32(0.1))
    off = (got.pre_bias.double() / (n * term) - 1).abs().max().item()
    assert off <= SUM, off
    # equal gradients of a layer norm's outputs give none to its input but for rounding: dR is dRn
    off = (got.post_bias.double() / (n * term * scale) - 1).abs().max().item()
    assert off <= SUM, off


def unit(x, eps=1e-5):
    x = x - x.mean(1, keepdim=True)
    return x * torch.rsqrt((x * x).mean(1, keepdim=True) + eps)


@pytest.mark.parametrize("n,F,act,stream,grad", [(2200003, 64, "f32", "f32", "f32"), (4300001, 64, "bf16", "bf16", "bf16"),
                                                 (1100001, 257, "f32", "bf16", "f32"), (140001, 1025, "bf16", "f32", "bf16"),
                                                 (70001, 4097, "f32", "f32", "f32"), (70001, 4096, "bf16", "bf16", "f32")])
@pytest.mark.parametrize("gate", ["col", "row", "full"])
def test_passes_in_parts(dg, device, n, F, act, stream, grad, gate):
    """Rows as in calls of their own, to the bit; column sums against float64."""
    types = {"f32": torch.float32, "bf16": torch.bfloat16}
    g = torch.Generator(device=device).manual_seed(n)
    make = lambda t, *s: torch.randn(*s, device=device, generator=g).to(types[t])  # noqa: E731
    Rn, B = make(stream, n, F), make(act, n, F)
    dZ, dRn = make(grad, n, F), make(stream, n, F)
    w = {k: 1.0 + 0.2 * make("f32", F) for k in ("post_weight", "post_bias", "pre_weight", "pre_bias")}
    shape = {"col": (F,), "row": (n, 1), "full": (n, F)}[gate]
    block = dict(w, gate=make(act if gate == "full" else "f32", *shape), scale=0.5, kind="layer")
    got = dg.norm_residual_backward(Rn, B, dZ, dRn, grad_bf16=grad == "bf16", **block)
    at = [0, n // 3, n // 2, n - 70]
    for a in at:
        rows = slice(a, a + 70)
        some = dict(block, gate=block["gate"] if gate == "col" else block["gate"][rows].contiguous())
        one = dg.norm_residual_backward(Rn[rows].contiguous(), B[rows].contiguous(), dZ[rows].contiguous(),
                                        dRn[rows].contiguous(), grad_bf16=grad == "bf16", **some)
        assert torch.equal(got.R[rows], one.R) and torch.equal(got.B[rows], one.B)
        if gate != "col":
            assert torch.equal(got.gate[rows], one.gate)
    # the vectors' gradients: d is dR (where the stream is float32: as it came), in float64
    if stream == "f32":
        sums, mags = {}, {}

        def add(name, t):
            sums[name] = sums.get(name, 0.0) + t.sum(0)
            mags[name] = mags.get(name, 0.0) + t.abs().sum(0)

        for a in range(0, n, 1 << 16):
            rows = slice(a, min(n, a + (1 << 16)))
            u2, u1, dz = unit(Rn[rows].double()), unit(B[rows].double()), dZ[rows].double()
            ga = block["gate"].double() if gate == "col" else block["gate"][rows].double()
            d = 0.5 * got.R[rows].double()
            add("pre_weight", dz * u2)
            add("pre_bias", dz)
            add("post_weight", d * ga * u1)
            add("post_bias", d * ga)
            if gate == "col":
                add("gate", d * (w["post_weight"].double() * u1 + w["post_bias"].double()))
        for name, want in sums.items():
            # a unit's magnitude bounds its error up to the mean's share: twice
            bound = 2 * SUM * mags[name] + ref.U * want.abs()
            off = (getattr(got, name).double() - want).abs()
            assert (off <= bound).all(), (name, (off / mags[name]).max().item())
    again = dg.norm_residual_backward(Rn, B, dZ, dRn, grad_bf16=grad == "bf16", **block)
    assert all(x is None or torch.equal(x, y) for x, y in zip(got, again))


def test_parts_in_a_graph(dg, device):
    n, F = 2200003, 64
    Rn, B, dZ = (torch.randn(n, F, device=device) for _ in range(3))
    w = torch.rand(F, device=device) + 0.5
    call = lambda: dg.norm_residual_backward(Rn, B, dZ, None, post_weight=w, pre_weight=w, gate=w)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cap = call()
    for k in range(3):
        dZ.mul_(1.5)
        eager = call()
        graph.replay()
        torch.cuda.synchronize()
        assert all(x is None or torch.equal(x, y) for x, y in zip(cap, eager))


# at least three steps of every workgroup, with two or more quads a thread (column sums in LDS; four: nothing ahead)
@pytest.mark.parametrize("n,F,act,stream,half", [(13000, 300, "f32", "f32", False), (7000, 512, "f32", "f32", False),
                                                 (7000, 700, "bf16", "f32", False), (7500, 1100, "f32", "f32", False),
                                                 (1700, 2048, "f32", "f32", False), (1700, 2051, "f32", "bf16", False),
                                                 (800, 5000, "f32", "f32", False), (800, 8191, "f32", "f32", False),
                                                 (800, 8192, "bf16", "bf16", True), (13000, 384, "bf16", "bf16", True),
                                                 (3400, 2048, "bf16", "bf16", True)])
def test_several_steps_of_wide_rows(dg, device, n, F, act, stream, half):
    c = _case(device, n, F, kind="layer", gate="col", act=act, stream=stream)
    _check_backward(dg, *c, grad_bf16=half)


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("stream", ["f32", "bf16"])
@pytest.mark.parametrize("half", [False, True])
def test_large_outputs(dg, device, act, stream, half):
    """Past 32 MiB the rows are stored past the L2s."""
    c = _case(device, 65541, 130, kind="layer", gate="col", act=act, stream=stream)
    _check_forward(dg, *c, norm_bf16=half)
    _check_backward(dg, *c, grad_bf16=half)
