"""C-ABI contract of the norms around a block, without a GPU: where an output replaces the one operand
that it may replace, no other operand may lie there too."""
import pytest

from conftest import gpu_available

pytestmark = pytest.mark.skipif(gpu_available(), reason="the addresses are no memory")

n, F = 10, 32
BYTES = n * F * 4


@pytest.fixture(scope="module")
def dg():
    import paper_2609_01983_amd as dg
    return dg


def at(k):
    return (1 << 30) + (k << 36)


def norm(dg, flags=0, gate=None, w1=None, b1=None, w2=None, b2=None):
    return dg.Norm(w1, b1, w2, b2, gate, 1e-5, 1.0, flags)


def test_forward_in_place(dg):
    R, B, Z, w, g = (at(k) for k in range(1, 6))
    layer = dg.NORM_POST | dg.NORM_LAYER

    def call(p, R=R, B=B, Rn=R, Z=Z):
        return dg.lib().dualgcn_norm_residual(p, R, B, Rn, Z, n, F, None)

    for p in (norm(dg), norm(dg, layer, w1=w, b1=w, w2=w, b2=w), norm(dg, dg.GATE_FULL, g)):
        assert call(p) == dg.ERR_NO_DEVICE
    bad = [(norm(dg, dg.NORM_POST, w1=R), {}), (norm(dg, layer, b1=R), {}), (norm(dg, w2=R), {}),
           (norm(dg, dg.NORM_LAYER, b2=R), {}), (norm(dg, dg.GATE_FEATURE, R), {}), (norm(dg, dg.GATE_NODE, R), {}),
           (norm(dg, dg.GATE_FULL, R), {}), (norm(dg), dict(B=R)), (norm(dg, dg.IN_BF16), dict(B=R)),
           (norm(dg, dg.NORM_POST, w1=R + 128), {}), (norm(dg, w2=R + BYTES - 4), {}), (norm(dg), dict(Z=R))]
    for p, k in bad:
        assert call(p, **k) == dg.ERR_INVALID_ARG, (p.flags, k)
    # R read only: the others may share its memory, as operands do
    assert call(norm(dg, dg.NORM_POST, w1=R, w2=R), Rn=at(9)) == dg.ERR_NO_DEVICE
    assert call(norm(dg), B=R, Rn=at(9)) == dg.ERR_NO_DEVICE


def test_backward_in_place(dg):
    Rn, B, dZ, d, dB, ws, g, w = (at(k) for k in range(1, 9))

    def call(flags=dg.NORM_POST | dg.NORM_LAYER | dg.GATE_FEATURE, Rn=Rn, B=B, dZ=dZ, gate=g, dR=d, **vectors):
        p = norm(dg, flags, gate, **vectors)
        return dg.lib().dualgcn_norm_residual_backward(p, Rn, B, dZ, d, dR, dB, None, n, F, ws, 1 << 20, None)

    assert call() == dg.ERR_NO_DEVICE and call(w1=w, b1=w, w2=w, b2=w) == dg.ERR_NO_DEVICE
    for k in (dict(w1=d), dict(b1=d), dict(w2=d), dict(b2=d), dict(gate=d), dict(dZ=d), dict(B=d), dict(Rn=d),
              dict(flags=dg.NORM_POST | dg.GATE_FULL, gate=d), dict(flags=dg.GATE_NODE, gate=d),
              dict(flags=dg.IN_BF16, gate=None, B=d), dict(w1=d + 128)):
        assert call(**k) == dg.ERR_INVALID_ARG, k
    for k in (dict(w1=d), dict(dZ=d), dict(B=d), dict(Rn=d)):
        assert call(dR=at(12), **k) == dg.ERR_NO_DEVICE, k
