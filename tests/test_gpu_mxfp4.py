"""The update phase from 4-bit operands on the GPU: the quantisers code for code against the definition, the product
against float64.

Product's tolerance, u = 2^-24: every product of two elements is exact, and the matrix cores add the F_in products of an
element in float32, each addition off by a rounding or a truncation (2 u) of at most the sum of magnitudes:
|T - exact| <= 2 u (F_in + 16) sum |x| |w|, and half a step more for T's own type.  Where the scales are alike, or
within 2^-2 .. 2^2 of each other, every sum is a multiple of a step of which 2^24 are not reached: then T is exact."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
TABLE = np.concatenate([GRID, -GRID])


@pytest.fixture(scope="module")
def dg(device):
    import paper_2609_01983_amd as dg
    return dg


def blocks(F):
    return -(-F // 32)


def quantised(X):
    """(codes [n, 32 blocks], scales [n, blocks]) of a float64 array, by comparisons."""
    n, F = X.shape
    pad = np.zeros((n, blocks(F) * 32))
    pad[:, :F] = X
    v = pad.reshape(n, -1, 32)
    bad = ~np.isfinite(v).all(2)
    amax = np.where(np.isfinite(v), np.abs(v), 0.0).max(2)
    # the least k with amax <= 7 * 2^k: amax / 7 = m 2^e with m in [0.5, 1), by exact comparisons
    _, e = np.frexp(amax / 7.0)
    k = np.where(amax <= np.ldexp(7.0, e - 1), e - 1, np.where(amax <= np.ldexp(7.0, e), e, e + 1))
    k = np.where(amax > 0, np.maximum(k, -127), 0)
    scale = np.where(bad, 255, k + 127)
    with np.errstate(invalid="ignore"):
        a = np.abs(v) * np.ldexp(1.0, -k)[:, :, None]
    code = np.zeros(a.shape, np.uint8)
    for j in range(7):
        mid = (GRID[j] + GRID[j + 1]) / 2
        code += (a >= mid) if j % 2 else (a > mid)
    code += 8 * np.signbit(v).astype(np.uint8)
    code[bad] = 0
    return code.reshape(n, -1), scale.astype(np.uint8)


def pack(code):
    return (code[:, ::2] | code[:, 1::2] << 4).astype(np.uint8)


def values(Q, scales):
    """float64 values of device (Q, scales)."""
    q = Q.cpu().numpy()
    c = np.stack([q & 15, q >> 4], 2).reshape(q.shape[0], -1)
    s = scales.cpu().numpy().astype(int)
    f = np.where(s == 255, np.nan, np.ldexp(1.0, s - 127))
    return TABLE[c] * np.repeat(f, 32, 1)


def same(Q, scales, want, what):
    code, s = want
    assert np.array_equal(scales.cpu().numpy(), s), f"{what}: scales"
    assert np.array_equal(Q.cpu().numpy(), pack(code)), f"{what}: codes"


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n,F", [(1, 1), (3, 2), (5, 3), (7, 4), (2, 31), (9, 32), (4, 33), (17, 200), (1000, 528), (3, 1024), (1, 70001),
                                 (4099, 40), (70000, 7), (2000, 96)])
def test_quantize(dg, device, n, F, bf16):
    rng = np.random.default_rng(n + F)
    X = torch.from_numpy((rng.standard_normal((n, F)) * np.exp(3 * rng.standard_normal((n, 1)))).astype(np.float32))
    X = (X.to(torch.bfloat16) if bf16 else X).to(device)
    Q, s = dg.quantize_mxfp4(X)
    same(Q, s, quantised(X.double().cpu().numpy()), f"{n} x {F}")
    for out_bf16 in (False, True):
        Y = dg.dequantize_mxfp4(Q, s, F, out_bf16=out_bf16)
        assert np.array_equal(Y.double().cpu().numpy(), values(Q, s)[:, :F])


def test_quantize_every_rounding(dg, device):
    """Numbers at and beside every middle between two codes, and beside the scale's own borders 7 * 2^k, with every scale that
    is a normal float32 number and some below."""
    mid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    f = np.float32
    some = np.concatenate([GRID, mid, np.nextafter(mid.astype(f), f(0)), np.nextafter(mid.astype(f), f(9))])
    assert some.size == 29
    rows = []
    for top in (6.0, 7.0, float(np.nextafter(f(7), f(0))), float(np.nextafter(f(7), f(9))), 3.6, float(np.nextafter(f(3.5), f(9)))):
        for sign in (1, -1):
            v = np.concatenate([some[some <= top], np.zeros(32)])[:30]
            rows.append(np.concatenate([sign * v, [top, -0.0]]))
    X = np.array(rows, np.float32)
    for shift in (0, 1, 30, -60, 100, 124, -100, -122, -126, -127, -130, -140):
        with np.errstate(over="ignore"):
            Y = torch.from_numpy(np.ldexp(X, shift).astype(np.float32)).to(device)
        for t in (Y, Y.to(torch.bfloat16)):
            Q, s = dg.quantize_mxfp4(t)
            same(Q, s, quantised(t.double().cpu().numpy()), f"shift {shift}")
    b = torch.arange(0, 1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    b = b[b.float().abs() <= 7].float()                  # every bfloat16 number of a block of scale 1
    b = torch.cat([b, torch.zeros(-b.numel() % 31)]).view(-1, 31)
    b = torch.cat([b, torch.full((b.shape[0], 1), 7.0)], 1).to(torch.bfloat16).to(device).contiguous()
    Q, s = dg.quantize_mxfp4(b)
    assert (s == 127).all()
    same(Q, s, quantised(b.double().cpu().numpy()), "bfloat16")


def test_quantize_zeros_infinities_nan_and_extremes(dg, device):
    X = torch.randn(9, 96, device=device)
    X[0] = 0.0
    X[1, 3], X[1, 50] = float("inf"), float("nan")
    X[2, :32] = float("-inf")
    X[3] = torch.finfo(torch.float32).max
    X[4] = 1e-40                                         # subnormal
    X[5] = 1e-45
    X[6] = -0.0
    X[7, 40:] = torch.finfo(torch.float32).tiny
    Q, s = dg.quantize_mxfp4(X)
    same(Q, s, quantised(X.double().cpu().numpy()), "extremes")
    Y = dg.dequantize_mxfp4(Q, s)
    assert torch.isnan(Y[1, :64]).all() and torch.isfinite(Y[1, 64:]).all() and torch.isnan(Y[2, :32]).all()
    assert (Y[0] == 0).all() and (Y[5] == 0).all() and torch.equal(torch.signbit(Y[6]), torch.signbit(X[6]))


def test_dequantize_every_value(dg, device):
    """All codes under all scales."""
    codes = np.tile(np.arange(32) % 16, (256, 1)).astype(np.uint8)
    Q = torch.from_numpy(pack(codes)).to(device)
    s = torch.arange(256, dtype=torch.uint8, device=device).view(256, 1)
    want = values(Q, s)
    for out_bf16 in (False, True):
        got = dg.dequantize_mxfp4(Q, s, out_bf16=out_bf16).double().cpu().numpy()
        finite = np.abs(want) < 2.0 ** 128
        assert np.array_equal(got[finite], want[finite]) and np.isnan(got[255]).all()
        over = ~finite & ~np.isnan(want)
        assert np.array_equal(got[over], np.sign(want[over]) * np.inf)


@pytest.mark.parametrize("F_in,F_out", [(1, 1), (3, 130), (32, 64), (33, 63), (128, 65), (256, 64), (1000, 333)])
def test_quantize_weight(dg, device, F_in, F_out):
    rng = np.random.default_rng(F_in)
    W = (rng.standard_normal((F_in, F_out)) * 0.1).astype(np.float32)
    Wd = torch.from_numpy(W).to(device)
    same(*dg.quantize_weight_mxfp4(Wd), quantised(np.ascontiguousarray(W.T).astype(np.float64)), "transposed")
    same(*dg.quantize_weight_mxfp4(Wd, transpose=False), quantised(W.astype(np.float64)), "as it stands")


def operands(device, n, F_in, F_out, spread=10, seed=0, tail=False):
    """Random codes and scales within 2^-spread .. 2^spread; tail: what lies behind F_in in X's last blocks is garbage, in W's 0."""
    rng = np.random.default_rng(seed + n + F_in + F_out)
    kb = blocks(F_in)

    def one(rows, clean):
        c = rng.integers(0, 16, (rows, 32 * kb)).astype(np.uint8)
        if clean:
            c[:, F_in:] = 0
        s = rng.integers(127 - spread, 128 + spread, (rows, kb)).astype(np.uint8)
        return [torch.from_numpy(t).to(device) for t in (pack(c), s)]

    return one(n, not tail) + one(F_out, True)


def product(Xq, sx, Wq, sw):
    """(exact, sum of magnitudes) as float64 on the device."""
    dev = Xq.device
    table = torch.tensor(TABLE, device=dev)

    def decode(Q, s):
        v = table[torch.stack([Q & 15, Q >> 4], 2).flatten(1).long()]
        return v * torch.exp2(s.double() - 127).repeat_interleave(32, 1)

    X, W = decode(Xq, sx), decode(Wq, sw).t().contiguous()
    return X @ W, X.abs() @ W.abs()


def check(dg, ops, out_bf16=False, exact=False, **more):
    T = dg.update_mxfp4(*ops, out_bf16=out_bf16, **more)
    want, mag = product(*ops)
    if exact:
        assert torch.equal(T, want.float().to(T.dtype)), "not exact"
        return T
    bound = 2 * U * (32 * ops[1].shape[1] + 16) * mag
    bound = bound + (2.0 ** -8 if out_bf16 else U) * (want.abs() + bound)
    bad = ~((T.double() - want).abs() <= bound)
    assert not bad.any(), f"{int(bad.sum())} outside, first at {bad.nonzero()[0].tolist()}"
    return T


SHAPES = [(1, 1), (16, 1), (32, 32), (100, 48), (128, 128), (144, 129), (256, 64), (256, 256), (528, 200), (1024, 256), (1056, 33), (4096, 130),
          (96, 700)]


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 33, 127, 128, 255, 256, 257, 513, 5000, 70001])
@pytest.mark.parametrize("F_in,F_out", SHAPES)
def test_update_is_exact_for_like_scales(dg, device, n, F_in, F_out):
    """Every element of every tile: scales within 2^-1 .. 2^1 of each other on each side."""
    if n * F_in * F_out > 3e10:
        n = 6000
    for out_bf16 in (False, True):
        check(dg, operands(device, n, F_in, F_out, spread=1, tail=True), out_bf16, exact=True)


@pytest.mark.parametrize("n,F_in,F_out", [(1, 8192, 100), (40, 1024, 256), (3000, 272, 130), (513, 2048, 513), (9000, 4096, 300), (70001, 96, 40)])
@pytest.mark.parametrize("out_bf16", [False, True])
def test_update(dg, device, n, F_in, F_out, out_bf16):
    check(dg, operands(device, n, F_in, F_out), out_bf16)
    check(dg, operands(device, n, F_in, F_out, spread=30), out_bf16)


@pytest.mark.parametrize("n,F_in,F_out", [(1, 256, 8192), (300, 128, 5001), (40000, 256, 1024), (3, 1024, 65536), (2, 65536, 3),
                                          (4096, 4096, 4096), (1000, 65536, 40), (2500, 3200, 2600)])
def test_wide(dg, device, n, F_in, F_out):
    check(dg, operands(device, n, F_in, F_out, spread=1), exact=32 * blocks(F_in) <= 7281)


def test_scales_far_from_each_other(dg, device):
    """2^-123 beside 2^123 multiply to 1; a scale of 0 is 2^-127; where products of 1/4 at least lie past float32's range
    (2^191 / 4) so does every partial sum, of either sign: the element is infinite or NaN."""
    for n, F_in, F_out in ((5, 96, 20), (700, 160, 70), (3000, 512, 300)):
        Xq, sx, Wq, sw = operands(device, n, F_in, F_out, spread=0)
        want = check(dg, (Xq, sx, Wq, sw), exact=True)
        assert torch.equal(dg.update_mxfp4(Xq, sx + 123, Wq, sw - 123), want)
        assert torch.equal(dg.update_mxfp4(Xq, sx - 127, Wq, sw + 127), want)
        got = dg.update_mxfp4(Xq, sx + 127, Wq, sw + 64)
        assert not torch.isfinite(got).any()
        assert (dg.update_mxfp4(Xq, sx - 127, Wq, sw - 100) == 0).all()


def test_rows_and_columns_do_not_mix(dg, device):
    """A NaN scale in one row of X reaches its row of T alone, one of W its column; the same bits whatever the others are."""
    for n, F_in, F_out in ((40, 272, 70), (3000, 272, 70), (3000, 2080, 520)):
        Xq, sx, Wq, sw = operands(device, n, F_in, F_out)
        clean = dg.update_mxfp4(Xq, sx, Wq, sw)
        sn = sx.clone()
        sn[n - 3, sx.shape[1] - 1] = 255
        T = dg.update_mxfp4(Xq, sn, Wq, sw)
        assert torch.isnan(T[n - 3]).all()
        T[n - 3] = clean[n - 3]
        assert torch.equal(T, clean)
        wn = sw.clone()
        wn[F_out - 1, 0] = 255
        T = dg.update_mxfp4(Xq, sx, Wq, wn)
        assert torch.isnan(T[:, F_out - 1]).all() and torch.equal(T[:, :F_out - 1], clean[:, :F_out - 1])


def test_reads_and_writes_only_its_own(dg, device):
    """T inside a larger buffer at odd elements; scales at odd bytes; X that is followed by NaN scales."""
    for n, F_in, F_out in ((5, 48, 7), (1000, 48, 7), (700, 144, 130), (5000, 1120, 515)):
        Xq, sx, Wq, sw = operands(device, n, F_in, F_out)
        want = dg.update_mxfp4(Xq, sx, Wq, sw)
        kb = blocks(F_in)
        bx = torch.full((n * kb + 40,), 255, dtype=torch.uint8, device=device)
        bw = torch.full((F_out * kb + 40,), 255, dtype=torch.uint8, device=device)
        ox, ow = bx[3:3 + n * kb].view(n, kb), bw[1:1 + F_out * kb].view(F_out, kb)
        ox.copy_(sx)
        ow.copy_(sw)
        for t in (torch.float32, torch.bfloat16):
            buf = torch.full((n * F_out + 9,), 5.0, device=device, dtype=t)
            T = buf[3:3 + n * F_out].view(n, F_out)
            dg.update_mxfp4(Xq, ox, Wq, ow, T=T, out_bf16=t == torch.bfloat16)
            assert torch.equal(T, want.to(t)) and (buf[:3] == 5).all() and (buf[3 + n * F_out:] == 5).all()


def test_a_layer_and_its_gradient_in_4_bits(dg, device):
    """Quantise, multiply, and the gradient G W^T from the weight's other layout, against the product of the numbers that
    the quantised operands stand for, and against the float32 product: an element is off by half a step at most, 1/4 of
    itself or 1/4 of its block's scale, which is at most 2/7 of the block's largest."""
    n, F_in, F_out = 3001, 160, 96
    X = torch.randn(n, F_in, device=device)
    W = torch.randn(F_in, F_out, device=device) * 0.1
    G = torch.randn(n, F_out, device=device)
    check(dg, [*dg.quantize_mxfp4(X), *dg.quantize_weight_mxfp4(W)])
    check(dg, [*dg.quantize_mxfp4(G), *dg.quantize_weight_mxfp4(W, transpose=False)])

    def error(t):
        b = t.double().abs().unflatten(1, (-1, 32))
        # below 1 half a step is 1/4 of the scale (at most 2/7 of the largest, more than 1/7); from 1 to 2 as well; then 1/4 of the element
        return torch.maximum(b / 4, (b.amax(2, keepdim=True) * 2 / 7 / 4).expand_as(b)).flatten(1)

    T = dg.update_mxfp4(*dg.quantize_mxfp4(X), *dg.quantize_weight_mxfp4(W)).double()
    Xe, We = error(X), error(W.t().contiguous()).t().contiguous()
    bound = Xe @ W.double().abs() + X.double().abs() @ We + Xe @ We + 1e-4
    assert ((T - X.double() @ W.double()).abs() <= bound).all()


def test_streams_and_graphs(dg, device):
    for n, F_in, F_out in ((3, 256, 128), (3000, 256, 128), (2000, 2048, 1024)):
        X = torch.randn(n, F_in, device=device)
        W = torch.randn(F_in, F_out, device=device)

        def call(stream=None):
            Xq, sx = dg.quantize_mxfp4(X, stream=stream)
            Wq, sw = dg.quantize_weight_mxfp4(W, stream=stream)
            return dg.update_mxfp4(Xq, sx, Wq, sw, out_bf16=True, stream=stream), dg.dequantize_mxfp4(Xq, sx, stream=stream)

        want = call()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = call(side)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cap = call()
        for _ in range(3):
            X.normal_()
            want = call()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(cap, want))


def test_more_than_2_to_the_31_elements(dg, device):
    n, F_in, F_out = (1 << 23) + 5, 272, 272
    Xb = torch.empty(n, F_in, device=device, dtype=torch.bfloat16).normal_()
    Q, s = dg.quantize_mxfp4(Xb)
    _, _, Wq, sw = operands(device, 1, F_in, F_out)
    rows = torch.tensor([0, 1 << 22, n - 2, n - 1], device=device)
    part = Xb[rows].contiguous()
    Qp, sp = dg.quantize_mxfp4(part)
    assert torch.equal(Q[rows], Qp) and torch.equal(s[rows], sp)
    assert torch.equal(dg.dequantize_mxfp4(Q, s, F_in, out_bf16=True)[rows], dg.dequantize_mxfp4(Qp, sp, F_in, out_bf16=True))
    del Xb
    T = dg.update_mxfp4(Q, s, Wq, sw, out_bf16=True)
    want = product(Qp, sp, Wq, sw)[0]
    assert ((T[rows].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -11 * want.abs().max()).all()


def test_more_rows_than_a_launch_takes(dg, device):
    """2^29 and some rows of one block: several launches, the last of a few rows."""
    n = (1 << 29) + 77
    Xq = torch.zeros(n, 16, dtype=torch.uint8, device=device)
    Xq[:, 0] = 0x21                                      # 0.5 and 1
    Xq[-1, 0], Xq[(1 << 29) - 1, 0] = 0x77, 0x65
    sx = torch.full((n, 1), 127, dtype=torch.uint8, device=device)
    sx[-2] = 130
    Wq = torch.zeros(1, 16, dtype=torch.uint8, device=device)
    Wq[0, 0] = 0x42                                      # 1 and 2
    sw = torch.full((1, 1), 128, dtype=torch.uint8, device=device)
    T = dg.update_mxfp4(Xq, sx, Wq, sw, out_bf16=True)[:, 0]
    special = {n - 1: 36.0, n - 2: 40.0, (1 << 29) - 1: 22.0}
    for row, want in special.items():
        assert T[row].item() == want
    T[list(special)] = 5.0
    assert (T == 5).all()


def test_refusals(dg, device):
    Xq, sx, Wq, sw = operands(device, 40, 64, 32)
    for bad in (lambda: dg.update_mxfp4(Xq.float(), sx, Wq, sw), lambda: dg.update_mxfp4(Xq.cpu(), sx, Wq, sw),
                lambda: dg.quantize_mxfp4(sx.double()), lambda: dg.update_mxfp4(Xq, sx.float(), Wq, sw)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: dg.update_mxfp4(Xq, sx[:39].contiguous(), Wq, sw), lambda: dg.update_mxfp4(Xq, sx, Wq[:, :16].contiguous(), sw),
                lambda: dg.update_mxfp4(Xq, sx, Wq[:, :16].contiguous(), sw[:, :1].contiguous()),
                lambda: dg.update_mxfp4(Xq[:, :24].contiguous(), sx, Wq, sw), lambda: dg.dequantize_mxfp4(Xq, sx, 32),
                lambda: dg.dequantize_mxfp4(Xq, sx, 65), lambda: dg.update_mxfp4(Xq, sx, Wq, sw, T=torch.empty(40, 31, device=device)),
                lambda: dg.quantize_mxfp4(torch.zeros(4, 4, device=device).t()[:, :3])):
        with pytest.raises(ValueError):
            bad()
    flat = torch.zeros(32 * 40 + 16, dtype=torch.uint8, device=device)
    with pytest.raises(dg.DualGCNError) as e:            # rows that are not 16-byte aligned
        dg.update_mxfp4(flat[1:1 + 32 * 40].view(40, 32), sx, Wq, sw)
    assert e.value.status == dg.ERR_INVALID_ARG
    with pytest.raises(dg.DualGCNError) as e:
        dg.quantize_mxfp4(torch.zeros(1, 1 << 20, device=device))
    assert e.value.status == dg.ERR_UNSUPPORTED
