"""Scales of the 8-bit operands from one end of float32 to the other: the result is right wherever it
is a float32 number, whatever the two scales' product is.

Tolerance, u = 2^-24, as in test_gpu_fp8.py: a block's products are summed with an error of at most 2 u 128 of their
magnitudes; the scales' product, its product with the sum and the sum over at most 8 blocks add at most
2 + 8 roundings.  Results below 2^-126 are rounded to multiples of 2^-149, half a step a block and sum; a bfloat16
below 2^-126 is a multiple of 2^-133 (2^-126 with 7 fraction bits), so storing one is off by up to 2^-134."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def dg(device):
    import paper_2609_01983_amd as dg
    return dg


def _operands(device, n, F_in, F_out, seed=0):
    g = torch.Generator().manual_seed(seed + n + F_in + F_out)
    Xq = (torch.randn(n, F_in, generator=g) * 60).clamp(-448, 448).to(E4M3)
    Wq = (torch.randn(F_out, F_in, generator=g) * 60).clamp(-448, 448).to(E4M3)
    return Xq.to(device), Wq.to(device)


def _check(dg, Xq, sx, Wq, sw, out_bf16=False):
    T = dg.update_fp8(Xq, sx, Wq, sw, out_bf16=out_bf16).double()
    F_out, F_in = Wq.shape
    want = mag = 0.0
    for b in range(sx.shape[1]):
        k = slice(128 * b, min(F_in, 128 * (b + 1)))
        s = sx[:, b:b + 1].double() * sw[:, b].double().repeat_interleave(128)[:F_out]
        X, W = Xq[:, k].double(), Wq[:, k].double()
        want = want + (X @ W.t().contiguous()) * s
        mag = mag + (X.abs() @ W.abs().t().contiguous()) * s.abs()
    bound = 2 * U * 144 * mag
    bound = bound + (2.0 ** -8 if out_bf16 else U) * (want.abs() + bound) + 24 * 2.0 ** -149
    bound = bound + (2.0 ** -134 if out_bf16 else 0.0)
    top = torch.finfo(torch.float32).max
    fine = mag < top / 4                                 # no partial sum overflows (the others are not looked at)
    bad = fine & ~((T - want).abs() <= bound)
    assert not bad.any(), (f"{int(bad.sum())} outside, first at {bad.nonzero()[0].tolist()}: "
                           f"{T[bad][0].item()} for {want[bad][0].item()}")


# few rows and many; narrow and wide; a short last block; columns across a border of 128
@pytest.mark.parametrize("n", [1, 37, 600, 3001])
@pytest.mark.parametrize("F_in,F_out", [(64, 32), (128, 130), (528, 200), (1024, 256)])
@pytest.mark.parametrize("sx,sw", [(1e30, 1e10), (1e10, 1e30), (3e-33, 1.7e-11), (1.7e-11, 3e-33), (1e-38, 1e30), (1e30, 1e-38),
                                   (3e38, 1e-38), (1e-30, 1e-30), (1e-44, 1e20), (7e30, 3e-30), (2.0 ** 120, 2.0 ** -126),
                                   (1.1e-19, 1.3e-19)])
def test_products_of_scales(dg, device, n, F_in, F_out, sx, sw):
    """All blocks have such scales, then one block or row of them among ordinary ones."""
    Xq, Wq = _operands(device, n, F_in, F_out)
    kb, nb = -(-F_in // 128), -(-F_out // 128)
    rng = np.random.default_rng(n + F_in)
    one = lambda *s: torch.from_numpy(rng.uniform(0.3, 1.0, s).astype(np.float32)).to(device)  # noqa: E731
    if sx * sw < 1e38 / 448 ** 2 / F_in:
        _check(dg, Xq, sx * one(n, kb), Wq, sw * one(nb, kb))
        _check(dg, Xq, sx * one(n, kb), Wq, sw * one(nb, kb), out_bf16=True)
    a, b = one(n, kb), one(nb, kb)
    a[n // 2] *= sx                                      # one row, whose products with the last columns need it
    b[-1] *= sw
    _check(dg, Xq, a, Wq, b)
    a, b = one(n, kb), one(nb, kb)
    a[:, -1] *= sx                                       # the last, short block
    b[:, -1] *= sw
    Z = Xq.float()
    Z[:, 128 * (kb - 1):] = 0.0                          # whose products sum to zero: no infinity times it
    _check(dg, Z.to(E4M3), a, Wq, b)


@pytest.mark.parametrize("n", [3, 600])
def test_scales_that_are_zero_infinite_or_nan(dg, device, n):
    Xq, Wq = _operands(device, n, 256, 40)
    sx, sw = torch.full((n, 2), 1e30, device=device), torch.full((1, 2), 1e-30, device=device)
    sx[0, 1] = 0.0
    sx[1, 0] = float("inf")
    sx[2, 1] = float("nan")
    T = dg.update_fp8(Xq, sx, Wq, sw)
    assert torch.isnan(T[2]).all() and not torch.isfinite(T[1]).any()
    keep = [v for v in range(n) if v not in (1, 2)]
    _check(dg, Xq.view(torch.uint8)[keep].view(E4M3), sx[keep].contiguous(), Wq, sw)
    sw[0, 0] = 0.0                                       # infinity times zero
    T = dg.update_fp8(Xq, sx, Wq, sw)
    assert torch.isnan(T[1]).all()
    _check(dg, Xq.view(torch.uint8)[keep].view(E4M3), sx[keep].contiguous(), Wq, sw)
