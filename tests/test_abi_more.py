"""C-ABI contract of the group norms over batches, the clipped gradients and the 4-bit update, without a GPU: every refusal
comes before a device is touched, and arguments that are in order report that there is none."""
import ctypes

import pytest

from conftest import gpu_available

pytestmark = pytest.mark.skipif(gpu_available(), reason="the addresses are no memory")


def at(k):
    """Operand k, far from the others and 256-byte aligned."""
    return (1 << 30) + (k << 36)


@pytest.fixture(scope="module")
def dg():
    import paper_2609_01983_amd as dg
    return dg


def group(dg, ptr=at(20), w=at(21), b=at(22), eps=1e-5, graphs=4, F=32, groups=4, flags=0):
    return dg.GroupNorm(ptr, w, b, eps, graphs, F, groups, flags)


PARAMETERS_OUT = [dict(F=0), dict(F=-4), dict(groups=0), dict(groups=5), dict(groups=64), dict(graphs=0), dict(eps=0.0), dict(eps=1e-40),
                  dict(eps=float("nan")), dict(eps=float("inf")), dict(flags=1 | 4096), dict(flags=1 << 20), dict(w=at(21) + 2),
                  dict(b=at(22) + 1), dict(ptr=at(20) + 2), dict(flags=16)]


def test_group_norm(dg):
    L = dg.lib()
    X, Y, st, ws = (at(k) for k in range(1, 5))
    need = ctypes.c_size_t()
    q = L.dualgcn_group_norm_act_workspace
    assert q(group(dg), 10, ctypes.byref(need)) == dg.OK and need.value == 0         # no graph can be long
    assert q(group(dg), 100000, ctypes.byref(need)) == dg.OK and need.value >= 4 * 4 * 16
    assert q(group(dg), 10, None) == dg.ERR_INVALID_ARG and q(group(dg), 0, ctypes.byref(need)) == dg.ERR_INVALID_ARG
    assert q(None, 10, ctypes.byref(need)) == dg.ERR_INVALID_ARG
    assert q(group(dg, F=8192, groups=1), (1 << 31) - (1 << 22), ctypes.byref(need)) == dg.OK

    def call(n=10, X=X, Y=Y, st=st, ws=ws, size=1 << 24, **k):
        return L.dualgcn_group_norm_act(group(dg, **k), X, Y, st, n, ws, size, None)

    for k in (dict(), dict(Y=X), dict(ptr=None, graphs=0), dict(w=None, b=None), dict(flags=dg.RELU), dict(flags=dg.SILU | dg.ZERO_REST),
              dict(flags=dg.IN_BF16 | dg.OUT_BF16, X=X + 2, Y=X + 2), dict(F=8192, groups=1, size=1 << 32), dict(F=1, groups=1, n=1),
              dict(F=3, groups=3), dict(X=X + 4, Y=Y + 4), dict(ws=None, size=0), dict(n=100000, size=1 << 32)):
        assert call(**k) == dg.ERR_NO_DEVICE, k
    for k in (dict(ws=None), dict(size=64), dict(ws=ws + 64), dict(Y=ws), dict(ws=X)):
        assert call(**{**dict(n=100000, size=1 << 32), **k}) == dg.ERR_INVALID_ARG, k
    for k in PARAMETERS_OUT + [dict(n=0), dict(n=-1), dict(X=None), dict(Y=None), dict(st=None),
                               dict(st=st + 8), dict(Y=X + 4), dict(Y=X, flags=dg.OUT_BF16), dict(Y=st), dict(Y=at(20)), dict(Y=at(21) - 8),
                               dict(st=X), dict(X=X + 2), dict(Y=Y + 1), dict(flags=dg.GRAD_BF16)]:
        assert call(**k) == dg.ERR_INVALID_ARG, k
    for k in (dict(F=8193, groups=1), dict(n=(1 << 31) - (1 << 22) + 1), dict(graphs=(1 << 30) + 1)):
        assert call(**k) == dg.ERR_UNSUPPORTED, k


def test_group_norm_backward(dg):
    L = dg.lib()
    X, dY, st, dX, dw, db, ws = (at(k) for k in range(1, 8))
    need = ctypes.c_size_t()
    q = L.dualgcn_group_norm_act_backward_workspace
    assert q(group(dg), 10, ctypes.byref(need)) == dg.OK and need.value >= 4 * 4 * 16
    assert q(group(dg, groups=3), 10, ctypes.byref(need)) == dg.ERR_INVALID_ARG

    def call(n=10, X=X, dY=dY, st=st, dX=dX, dw=dw, db=db, ws=ws, size=1 << 24, **k):
        return L.dualgcn_group_norm_act_backward(group(dg, **k), X, dY, st, dX, dw, db, n, ws, size, None)

    for k in (dict(), dict(dX=dY), dict(dX=None), dict(dw=None), dict(db=None), dict(dX=None, dw=None, db=None), dict(ptr=None),
              dict(flags=dg.SILU | dg.OUT_BF16 | dg.GRAD_BF16 | dg.IN_BF16), dict(w=None, b=None)):
        assert call(**k) == dg.ERR_NO_DEVICE, k
    for k in PARAMETERS_OUT + [dict(n=0), dict(X=None), dict(dY=None), dict(st=None), dict(ws=None), dict(size=64), dict(ws=ws + 128),
                               dict(st=st + 8), dict(dX=X), dict(dX=dY + 4), dict(dw=db), dict(dw=dX), dict(db=st), dict(dX=ws), dict(dw=at(21)),
                               dict(dw=dw + 2), dict(dY=dY + 2)]:
        assert call(**k) == dg.ERR_INVALID_ARG, k
    assert call(F=8193, groups=1) == dg.ERR_UNSUPPORTED


def test_clipped_gradients(dg):
    L = dg.lib()
    norm, ws = at(30), at(31)
    need = ctypes.c_size_t()
    q = L.dualgcn_grad_norm_workspace
    assert q(1, ctypes.byref(need)) == dg.OK and q(1 << 20, ctypes.byref(need)) == dg.OK and need.value <= 1 << 28
    assert q(0, ctypes.byref(need)) == dg.ERR_INVALID_ARG and q(3, None) == dg.ERR_INVALID_ARG
    assert q((1 << 20) + 1, ctypes.byref(need)) == dg.ERR_UNSUPPORTED

    def rows(*tensors):
        out = (dg.Grad * max(1, len(tensors)))()
        for i, t in enumerate(tensors):
            out[i] = dg.Grad(*t)
        return out

    g, w, o = [at(k) for k in (1, 2, 3)], [at(k) for k in (4, 5, 6)], [at(k) for k in (7, 8, 9)]
    BF = dg.GRAD_BF16

    def norm_of(*t, tensors=None, norm=norm, ws=ws, size=1 << 20):
        return L.dualgcn_grad_norm(rows(*t), len(t) if tensors is None else tensors, norm, ws, size, None)

    def clip(*t, most=1.0, eps=1e-6, norm=norm, ws=ws, size=1 << 20):
        return L.dualgcn_clip_grads(rows(*t), len(t), most, eps, norm, ws, size, None)

    def step(*t, most=1.0, eps=1e-6, lr=0.1):
        return L.dualgcn_clipped_sgd(rows(*t), len(t), most, eps, lr, norm, ws, 1 << 20, None)

    no = None
    assert norm_of((g[0], no, no, 10, 0), (g[1] + 2, no, no, 7, BF), (g[0], no, no, 10, 0), (no, no, no, 0, 0)) == dg.ERR_NO_DEVICE
    for t in ([(no, no, no, 5, 0)], [(g[0] + 2, no, no, 5, 0)], [(g[0] + 1, no, no, 5, BF)], [(g[0], no, no, -1, 0)], [(g[0], no, no, 5, 1)],
              [(g[0], w[0], no, 5, 0)], [(g[0], no, o[0], 5, 0)], [(norm, no, no, 5, 0)], [(ws + 64, no, no, 5, 0)]):
        assert norm_of(*t) == dg.ERR_INVALID_ARG, t
    one = (g[0], no, no, 5, 0)
    for k in (dict(tensors=0), dict(tensors=-1), dict(norm=None), dict(norm=norm + 2), dict(ws=None), dict(ws=ws + 8), dict(size=100),
              dict(norm=ws)):
        assert norm_of(one, **k) == dg.ERR_INVALID_ARG, k
    assert norm_of((g[0], no, no, (1 << 40) + 1, 0)) == dg.ERR_UNSUPPORTED
    assert L.dualgcn_grad_norm(None, 1, norm, ws, 1 << 20, None) == dg.ERR_INVALID_ARG

    for t in ([(g[0], no, g[0], 10, 0), (g[1], no, o[1], 10, BF)], [(no, no, no, 0, 0)], [(g[0], no, g[0], 10, 0), (g[0] + 40, no, g[0] + 40, 10, 0)]):
        assert clip(*t) == dg.ERR_NO_DEVICE, t
        for k in (dict(most=0.0), dict(most=float("inf")), dict(eps=0.0)):
            assert clip(*t, **k) == dg.ERR_NO_DEVICE
        for k in (dict(most=-1.0), dict(most=float("nan")), dict(eps=-1e-9), dict(eps=float("inf")), dict(eps=float("nan"))):
            assert clip(*t, **k) == dg.ERR_INVALID_ARG, k
    for t in ([(g[0], no, no, 10, 0)], [(g[0], w[0], o[0], 10, 0)], [(g[0], no, g[0] + 4, 10, 0)], [(g[0], no, g[0], 10, 0)] * 2,
              [(g[0], no, o[0], 10, 0), (g[1], no, o[0] + 36, 10, 0)], [(g[0], no, g[1], 10, 0), (g[1], no, g[0], 10, 0)],
              [(g[0], no, g[0], 10, 0), (g[0] + 36, no, o[0], 10, 0)], [(g[0], no, norm, 1, 0)], [(g[0], no, ws, 1, 0)],
              [(g[0], no, o[0] + 2, 10, 0)]):
        assert clip(*t) == dg.ERR_INVALID_ARG, t

    for t in ([(g[0], w[0], w[0], 10, 0), (g[1], w[1], o[1], 10, BF)], [(g[0], w[0], w[0], 9, 0), (g[0], w[1], w[1], 9, 0)], [(no, no, no, 0, 0)],
              [(g[0], w[0], o[0], 9, 0), (g[1], w[0], o[1], 9, 0)]):
        assert step(*t) == dg.ERR_NO_DEVICE, t
    for t in ([(g[0], no, o[0], 10, 0)], [(g[0], w[0], no, 10, 0)], [(g[0], w[0], g[0], 10, 0)], [(g[0], w[0], w[0], 9, 0), (g[1], w[0], o[1], 9, 0)],
              [(g[0], w[0], w[0] + 4, 9, 0)], [(g[0], w[0] + 2, o[0], 9, 0)], [(g[0], w[0], o[0] + 2, 9, BF)]):
        assert step(*t) == dg.ERR_INVALID_ARG, t
    for k in (dict(lr=float("nan")), dict(lr=float("inf")), dict(most=-2.0)):
        assert step((g[0], w[0], w[0], 10, 0), **k) == dg.ERR_INVALID_ARG


def test_clipped_gradients_of_too_many_elements(dg):
    # one gradient listed often has more chunks of it than a launch's partial sums have places for
    def call(times, count):
        t = (dg.Grad * times)(*[dg.Grad(at(1), None, None, count, 0) for _ in range(times)])
        return dg.lib().dualgcn_grad_norm(t, times, at(40), at(41), 1 << 20, None)

    assert call(5, 1 << 38) == dg.ERR_NO_DEVICE and call(160, 1 << 34) == dg.ERR_NO_DEVICE
    assert call(200, 1 << 36) == dg.ERR_UNSUPPORTED and call(9, 1 << 39) == dg.ERR_UNSUPPORTED
    assert call(8, 1 << 39) == dg.ERR_NO_DEVICE


def test_mxfp4(dg):
    L = dg.lib()
    X, Q, s, W, sw, T = (at(k) for k in range(1, 7))

    def quantize(X=X, n=10, F=40, flags=0, Q=Q, s=s):
        return L.dualgcn_quantize_mxfp4(X, n, F, flags, Q, s, None)

    def back(Q=Q, s=s, n=10, F=40, flags=0, X=X):
        return L.dualgcn_dequantize_mxfp4(Q, s, n, F, flags, X, None)

    for f, bf in ((quantize, dg.IN_BF16), (back, dg.OUT_BF16)):
        for k in (dict(), dict(flags=bf, X=X + 2), dict(F=1, n=1), dict(F=(1 << 20) - 1), dict(s=s + 1), dict(X=X + 4)):
            assert f(**k) == dg.ERR_NO_DEVICE, k
        for k in (dict(X=None), dict(Q=None), dict(s=None), dict(n=0), dict(F=0), dict(flags=8), dict(Q=Q + 8), dict(X=X + 2), dict(X=X + 1, flags=bf),
                  dict(X=Q), dict(X=s - 4)):
            assert f(**k) == dg.ERR_INVALID_ARG, k
        for k in (dict(F=1 << 20), dict(n=(1 << 31) - 1, F=65)):
            assert f(**k) == dg.ERR_UNSUPPORTED, k
    assert quantize(s=Q + 10 * 32) == dg.ERR_NO_DEVICE and back(s=Q) == dg.ERR_NO_DEVICE      # operands may share bytes
    for k in (dict(Q=s), dict(s=Q + 10 * 32 - 1)):
        assert quantize(**k) == dg.ERR_INVALID_ARG, k

    def weight(W=W, a=40, b=50, t=1, Q=Q, s=s):
        return L.dualgcn_quantize_weight_mxfp4(W, a, b, t, Q, s, None)

    for k in (dict(), dict(t=0), dict(a=1, b=1), dict(a=65536, b=65536)):
        assert weight(**k) == dg.ERR_NO_DEVICE, k
    for k in (dict(W=None), dict(Q=None), dict(s=None), dict(a=0), dict(b=-1), dict(Q=Q + 4), dict(W=W + 2), dict(Q=W), dict(s=W + 40 * 50 * 4 - 1)):
        assert weight(**k) == dg.ERR_INVALID_ARG, k
    assert weight(a=65537) == dg.ERR_UNSUPPORTED and weight(b=65537) == dg.ERR_UNSUPPORTED

    def update(X=Q, sx=s, W=W, sw=sw, T=T, n=10, a=40, b=50, flags=0):
        return L.dualgcn_update_mxfp4(X, sx, W, sw, T, n, a, b, flags, None)

    for k in (dict(), dict(flags=dg.OUT_BF16, T=T + 2), dict(n=1, a=1, b=1), dict(a=65536, b=65536), dict(T=T + 4), dict(sx=s + 3, sw=sw + 1)):
        assert update(**k) == dg.ERR_NO_DEVICE, k
    for k in (dict(X=None), dict(sx=None), dict(W=None), dict(sw=None), dict(T=None), dict(n=0), dict(a=0), dict(b=0), dict(flags=dg.IN_BF16),
              dict(X=Q + 8), dict(W=W + 4), dict(T=T + 2), dict(T=Q), dict(T=s - 4), dict(T=W + 50 * 32 - 4), dict(T=sw)):
        assert update(**k) == dg.ERR_INVALID_ARG, k
    for k in (dict(a=65537), dict(b=65537)):
        assert update(**k) == dg.ERR_UNSUPPORTED, k
