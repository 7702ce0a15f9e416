"""The update phase from 8-bit operands on the GPU: the quantisers bit for bit against torch's own
conversion, the product against float64.

Product's tolerance, u = 2^-24: the matrix cores sum a block's 128 products in float32 (each
product of two e4m3 numbers, widened to bfloat16, is exact), at most 128 roundings or truncations
(2 u each) of the sum of magnitudes; the two scales' product, the fma and the sum over at most 8 blocks add 2 + 8.  So
|T - exact| <= 2 u (128 + 16) sum |x| |w|; a bfloat16 T is off by another 2^-8 of itself."""
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


def _scale(amax):
    """The least power of two >= amax / 448, as the header defines it, in float64 (exact)."""
    amax = amax.astype(np.float64)
    out = np.ones_like(amax)
    some = amax > 0
    m, e = np.frexp(amax[some])
    out[some] = np.ldexp(1.0, np.maximum(np.where(m > 0.875, e - 8, e - 9), -126))
    return out


def _quantised(X, rows_per_block=1):
    """(e4m3 values as float64 (NaN for what is not finite), scales) of a float64 array."""
    n, F = X.shape
    nb, fb = -(-n // rows_per_block), -(-F // 128)
    pad = np.zeros((nb * rows_per_block, fb * 128))
    pad[:n, :F] = np.where(np.isfinite(X), np.abs(X), 0.0)
    amax = pad.reshape(nb, rows_per_block, fb, 128).max((1, 3))
    s = _scale(amax)
    full = np.repeat(np.repeat(s, 128, 1), rows_per_block, 0)[:n, :F]
    with np.errstate(invalid="ignore"):
        v = X / full
    v = np.where(np.isfinite(v), v, np.nan)
    # |v| <= 448 is a float32 (X is one and the scale a power of two) unless it is below 2^-126,
    # where both round to 0
    q = torch.from_numpy(v.astype(np.float32)).to(E4M3).double().numpy()
    return q, s


def _same(Q, s, want, what):
    q, ws = want
    got = Q.cpu().double().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(q)), what
    assert np.array_equal(np.nan_to_num(got), np.nan_to_num(q)), what
    assert np.array_equal(s.double().cpu().numpy(), ws), what


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n,F", [(1, 1), (3, 2), (5, 3), (7, 4), (2, 127), (9, 128), (4, 129), (17, 200), (1000, 528),
                                 (3, 1024), (1, 70001), (4099, 33)])
def test_quantize(dg, device, n, F, bf16):
    rng = np.random.default_rng(n + F)
    X = torch.from_numpy((rng.standard_normal((n, F)) * np.exp(3 * rng.standard_normal((n, 1)))).astype(np.float32))
    X = (X.to(torch.bfloat16) if bf16 else X).to(device)
    Q, s = dg.quantize_fp8(X)
    _same(Q, s, _quantised(X.double().cpu().numpy()), f"{n} x {F}")


def test_quantize_every_rounding(dg, device):
    """All bfloat16 numbers of a block's range against torch's rounding, and float32 numbers at and
    beside every border between two e4m3 numbers, subnormal ones among them."""
    e4 = torch.arange(0, 127, dtype=torch.uint8).view(E4M3).float().numpy().astype(np.float64)
    mid = (e4[1:] + e4[:-1]) / 2
    some = np.concatenate([e4, mid, np.nextafter(mid.astype(np.float32), np.float32(0)).astype(np.float64),
                           np.nextafter(mid.astype(np.float32), np.float32(1e9)).astype(np.float64)])
    some = np.concatenate([some, -some])
    rows = []
    for a in range(0, some.size, 127):                   # 448 at the end of each block: the scale is 1
        rows.append(np.concatenate([some[a:a + 127], np.zeros(127 - some[a:a + 127].size), [448.0]]))
    X = torch.from_numpy(np.array(rows, dtype=np.float32)).to(device)
    for shift in (0, 30, -60, 100):
        Y = X * 2.0 ** shift
        Q, s = dg.quantize_fp8(Y)
        assert (s == 2.0 ** shift).all()
        _same(Q, s, _quantised(Y.double().cpu().numpy()), f"shift {shift}")
    b = torch.arange(0, 1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    b = b[b.float().abs() <= 448].float()
    b = torch.cat([b, torch.zeros(-b.numel() % 127)]).view(-1, 127)
    b = torch.cat([b, torch.full((b.shape[0], 1), 448.0)], 1).to(torch.bfloat16).to(device).contiguous()
    Q, s = dg.quantize_fp8(b)
    _same(Q, s, _quantised(b.double().cpu().numpy()), "bfloat16")


def test_quantize_zeros_infinities_nan_and_extremes(dg, device):
    X = torch.randn(8, 256, device=device)
    X[0] = 0.0
    X[1, 3], X[1, 200] = float("inf"), float("nan")
    X[2, :128] = float("-inf")
    X[3] = torch.finfo(torch.float32).max
    X[4] = 1e-40                                         # subnormal
    X[5, 0] = 449.0
    X[6, 0] = 448.0
    Q, s = dg.quantize_fp8(X)
    _same(Q, s, _quantised(X.double().cpu().numpy()), "extremes")
    assert (s[0] == 1).all() and s[2, 0] == 1 and torch.isnan(Q[2, :128].float()).all()


@pytest.mark.parametrize("F_in,F_out", [(1, 1), (3, 130), (128, 128), (129, 127), (256, 64), (1000, 333)])
def test_quantize_weight(dg, device, F_in, F_out):
    rng = np.random.default_rng(F_in)
    W = rng.standard_normal((F_in, F_out)).astype(np.float32) * 0.1
    Wd = torch.from_numpy(W).to(device)
    Q, s = dg.quantize_weight_fp8(Wd)
    _same(Q, s, _quantised(np.ascontiguousarray(W.T).astype(np.float64), 128), "transposed")
    Q2, s2 = dg.quantize_weight_fp8(Wd, transpose=False)
    _same(Q2, s2, _quantised(W.astype(np.float64), 128), "as it stands")
    assert torch.equal(Q2.view(torch.uint8).t(), Q.view(torch.uint8)) and torch.equal(s2.t(), s)


def _operands(device, n, F_in, F_out, seed=0):
    g = torch.Generator().manual_seed(seed + n + F_in + F_out)
    Xq = (torch.randn(n, F_in, generator=g) * 60).clamp(-448, 448).to(E4M3)
    Wq = (torch.randn(F_out, F_in, generator=g) * 60).clamp(-448, 448).to(E4M3)
    kb, nb = -(-F_in // 128), -(-F_out // 128)
    sx = torch.rand(n, kb, generator=g) + 0.01           # any float32 numbers, no powers of two
    sw = torch.rand(nb, kb, generator=g) - 0.3
    return [t.to(device) for t in (Xq, sx, Wq, sw)]


def _exact(Xq, sx, Wq, sw):
    F_out, F_in = Wq.shape
    X = Xq.double() * sx.double().repeat_interleave(128, 1)[:, :F_in]
    W = Wq.double() * sw.double().repeat_interleave(128, 1)[:, :F_in].repeat_interleave(128, 0)[:F_out]
    return X @ W.t(), X.abs() @ W.abs().t()


def _check(dg, ops, out_bf16=False, **more):
    T = dg.update_fp8(*ops, out_bf16=out_bf16, **more)
    want, mag = _exact(*ops)
    bound = 2 * U * 144 * mag
    bound += (2.0 ** -8 if out_bf16 else U) * (want.abs() + bound)
    bad = ~((T.double() - want).abs() <= bound)
    assert not bad.any(), f"{int(bad.sum())} outside, first at {bad.nonzero()[0].tolist()}"
    return T


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 33, 255, 256, 257, 513, 5000, 70001])
@pytest.mark.parametrize("F_in,F_out", [(16, 1), (32, 32), (112, 48), (128, 128), (144, 129), (256, 64), (528, 200),
                                        (1024, 256), (1008, 33)])
@pytest.mark.parametrize("out_bf16", [False, True])
def test_update_fp8(dg, device, n, F_in, F_out, out_bf16):
    _check(dg, _operands(device, n, F_in, F_out), out_bf16)


# rows around the point from which the slices of a row tile share an XCD, in numbers that are no
# multiple of eight tiles
@pytest.mark.parametrize("n", [500, 512, 1793, 16128, 16640, 18433])
@pytest.mark.parametrize("F_in,F_out", [(256, 300), (1024, 161)])
def test_shared_slices(dg, device, n, F_in, F_out):
    _check(dg, _operands(device, n, F_in, F_out))


@pytest.mark.parametrize("n,F_in,F_out", [(1, 256, 8192), (300, 128, 5001), (40000, 256, 1024), (3, 1024, 65536)])
def test_wide_outputs(dg, device, n, F_in, F_out):
    _check(dg, _operands(device, n, F_in, F_out))


def test_rows_and_columns_do_not_mix(dg, device):
    """NaN in one row of X reaches its row of T alone, NaN in one row of W its column; the same
    bits whatever the other rows are; and whole rows of zeros and scales of zero."""
    for n in (40, 3000):
        Xq, sx, Wq, sw = _operands(device, n, 272, 70)
        clean = dg.update_fp8(Xq, sx, Wq, sw)
        Xn, Wn = Xq.clone(), Wq.clone()
        Xn.view(torch.uint8)[n - 3, 271] = 0x7F
        T = dg.update_fp8(Xn, sx, Wq, sw)
        assert torch.isnan(T[n - 3]).all()
        T[n - 3] = clean[n - 3]
        assert torch.equal(T, clean)
        Wn.view(torch.uint8)[69, 0] = 0xFF
        T = dg.update_fp8(Xq, sx, Wn, sw)
        assert torch.isnan(T[:, 69]).all() and torch.equal(T[:, :69], clean[:, :69])
        s0 = sx.clone()
        s0[2] = 0.0
        assert (dg.update_fp8(Xq, s0, Wq, sw)[2] == 0).all()


def test_reads_and_writes_only_its_own(dg, device):
    """T inside a larger buffer: nothing before or behind it is written; a T at odd elements."""
    for n, F_in, F_out in ((5, 48, 7), (1000, 48, 7), (700, 144, 130)):
        Xq, sx, Wq, sw = _operands(device, n, F_in, F_out)
        want = dg.update_fp8(Xq, sx, Wq, sw)
        for t in (torch.float32, torch.bfloat16):
            buf = torch.full((n * F_out + 9,), 5.0, device=device, dtype=t)
            T = buf[3:3 + n * F_out].view(n, F_out)
            dg.update_fp8(Xq, sx, Wq, sw, T=T, out_bf16=t == torch.bfloat16)
            assert torch.equal(T, want.to(t)) and (buf[:3] == 5).all() and (buf[3 + n * F_out:] == 5).all()


def test_a_layer_and_its_gradient_in_8_bits(dg, device):
    """Quantise, multiply, and the gradient G W^T from the weight's other layout, against the
    product of the numbers that the quantised operands stand for."""
    n, F_in, F_out = 3001, 160, 96
    X = torch.randn(n, F_in, device=device)
    W = torch.randn(F_in, F_out, device=device) * 0.1
    G = torch.randn(n, F_out, device=device)
    _check(dg, [*dg.quantize_fp8(X), *dg.quantize_weight_fp8(W)])
    _check(dg, [*dg.quantize_fp8(G), *dg.quantize_weight_fp8(W, transpose=False)])
    # against the float32 product: an operand's element is off by half a step, 2^-4 of itself (or
    # 2^-10 of its block's scale, its subnormal step)
    T = dg.update_fp8(*dg.quantize_fp8(X), *dg.quantize_weight_fp8(W)).double()
    small = 2.0 ** -10 * 2.0 ** -7                       # half the subnormal step over the largest, 448 > 2^8 / 2
    Xm = X.double().abs() * 2 ** -4 + small * X.double().abs().amax()
    Wm = W.double().abs() * 2 ** -4 + small * W.double().abs().amax()
    bound = Xm @ W.double().abs() + X.double().abs() @ Wm + Xm @ Wm + 1e-4
    assert ((T - X.double() @ W.double()).abs() <= bound).all()


def test_streams_and_graphs(dg, device):
    for n in (3, 3000):
        X = torch.randn(n, 256, device=device)
        W = torch.randn(256, 128, device=device)

        def call(stream=None):
            Xq, sx = dg.quantize_fp8(X, stream=stream)
            Wq, sw = dg.quantize_weight_fp8(W, stream=stream)
            return dg.update_fp8(Xq, sx, Wq, sw, out_bf16=True, stream=stream)

        want = call()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = call(side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cap = call()
        for _ in range(3):
            X.normal_()
            want = call()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(cap, want)


def test_more_than_2_to_the_31_elements(dg, device):
    n, F_in, F_out = (1 << 23) + 5, 272, 272
    Xq = torch.randint(0, 0x7F, (n, F_in), device=device, dtype=torch.uint8)
    sx = torch.rand(n, 3, device=device)
    _, _, Wq, sw = _operands(device, 1, F_in, F_out)
    Xq = Xq.view(E4M3)
    T = dg.update_fp8(Xq, sx, Wq, sw, out_bf16=True)
    rows = torch.tensor([0, 1 << 22, n - 2, n - 1], device=device).repeat(100)
    want = dg.update_fp8(Xq.view(torch.uint8)[rows].view(E4M3), sx[rows], Wq, sw, out_bf16=True)
    assert torch.equal(T[rows], want)
    del T
    Xb = torch.zeros(n, F_in, device=device, dtype=torch.bfloat16)
    Xb[-1] = 3.0
    Q, s = dg.quantize_fp8(Xb)
    assert (Q[-1].float() * s[-1, 0] == 3).all() and (Q[-2].float() == 0).all()


def test_refusals(dg, device):
    Xq, sx, Wq, sw = _operands(device, 40, 64, 32)
    with pytest.raises(TypeError):
        dg.update_fp8(Xq.float(), sx, Wq, sw)
    with pytest.raises(TypeError):
        dg.update_fp8(Xq.cpu(), sx, Wq, sw)
    with pytest.raises(ValueError):
        dg.update_fp8(Xq, sx[:39].contiguous(), Wq, sw)
    with pytest.raises(ValueError):
        dg.update_fp8(Xq, sx, Wq[:, :32].contiguous(), sw)
    with pytest.raises(ValueError):
        dg.update_fp8(Xq, sx, Wq, sw, T=torch.empty(40, 31, device=device))
    with pytest.raises(TypeError):
        dg.quantize_fp8(sx.double())
    with pytest.raises(ValueError):
        dg.quantize_fp8(sx.t().expand(3, 40))
    for F_in in (24, 1040):
        with pytest.raises(dg.DualGCNError) as e:
            dg.update_fp8(*_operands(device, 4, F_in, 16))
        assert e.value.status == dg.ERR_UNSUPPORTED
    flat = torch.zeros(64 * 40 + 16, dtype=torch.uint8, device=device)
    with pytest.raises(dg.DualGCNError) as e:            # rows that are not 16-byte aligned
        dg.update_fp8(flat[1:1 + 64 * 40].view(40, 64).view(E4M3), sx, Wq, sw)
    assert e.value.status == dg.ERR_INVALID_ARG
