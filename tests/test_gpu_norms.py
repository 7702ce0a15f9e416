"""The norms around a block on the GPU against float64 (normref.py, whose bounds are derived
there): every width class and its borders, types, gates, norms left out; gradients against the
formulas and against differences; rows of zeros, infinities and NaN; streams, graphs, refusals."""
import numpy as np
import pytest
import torch

import normref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dg(device):
    import paper_2609_01983_amd as dg
    return dg


def _case(device, n, F, kind="rms", post=True, pre=True, block=True, gate="none", sigmoid=False, act="f32",
          stream="f32", vectors=True, seed=0):
    """(device operands, float64 operands, keyword arguments for each)."""
    rng = np.random.default_rng(seed * 1000003 + n * 8209 + F)
    types = {"f32": torch.float32, "bf16": torch.bfloat16}

    def make(a, t):
        d = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(device).to(types[t])
        return d, d.double().cpu().numpy()

    size = np.exp(rng.standard_normal((n, 1)))
    dev, hst = {}, {}
    dev["R"], hst["R"] = make(rng.standard_normal((n, F)) * size + 0.3, stream)
    dev["B"], hst["B"] = make(rng.standard_normal((n, F)) * size[::-1] - 0.2, act) if block else (None, None)
    dev["dZ"], hst["dZ"] = make(rng.standard_normal((n, F)), "f32") if pre else (None, None)
    dev["dRn"], hst["dRn"] = make(rng.standard_normal((n, F)), stream)
    kd = dict(post_norm=post, pre_norm=pre, gate_sigmoid=sigmoid, scale=0.7, kind=kind, eps=1e-5)
    kh = dict(kd)
    for name, want, about in (("post_weight", post, 1.0), ("post_bias", post and kind == "layer", 0.0),
                              ("pre_weight", pre, 1.0), ("pre_bias", pre and kind == "layer", 0.0)):
        kd[name], kh[name] = make(about + 0.3 * rng.standard_normal(F), "f32") if want and vectors else (None, None)
    shape = {"none": None, "col": (F,), "row": (n, 1), "full": (n, F)}[gate]
    kd["gate"], kh["gate"] = (None, None) if shape is None else make(0.5 + rng.standard_normal(shape),
                                                                    act if gate == "full" else "f32")
    if gate == "row" and F == 1:
        kd["gate"] = kd["gate"].to(dev["B"].dtype)
        kh["gate"] = kd["gate"].double().cpu().numpy()
    return dev, hst, kd, kh


def _near(got, want, bound, what):
    half = ref.BF16 * (np.abs(want) + bound) if got.dtype == torch.bfloat16 else ref.U * np.abs(want)
    g = got.double().cpu().numpy()
    off = np.abs(g - want)
    bad = ~(off <= bound + half)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} outside; at {i} got {g[i]!r} want {want[i]!r} "
                             f"bound {(bound + half)[i]!r}")


def _check_forward(dg, dev, hst, kd, kh, **more):
    Rn, Z = dg.norm_residual(dev["R"], dev["B"], **kd, **more)
    if dev["B"] is not None:
        assert Rn.dtype == dev["R"].dtype
        _near(Rn, *ref.forward_stream(hst["R"], hst["B"], kh), "Rn")
    else:
        assert Rn is dev["R"]
    if kd["pre_norm"]:
        # from the stream as the device stored it
        _near(Z, *ref.forward_norm(Rn.double().cpu().numpy(), kh), "Z")
    else:
        assert Z is None
    return Rn, Z


def _check_backward(dg, dev, hst, kd, kh, grad_bf16=False):
    dZ, hZ = dev["dZ"], hst["dZ"]
    if grad_bf16 and dZ is not None:
        dZ = dZ.to(torch.bfloat16)
        hZ = dZ.double().cpu().numpy()
    got = dg.norm_residual_backward(dev["R"], dev["B"], dZ, dev["dRn"], grad_bf16=grad_bf16, **kd)
    want = ref.backward(hst["R"], hst["B"], hZ, hst["dRn"], kh)
    for name in dg.NormGrads._fields:
        g = getattr(got, name)
        if name in ("post_weight", "post_bias", "pre_weight", "pre_bias") and kd[name] is None:
            assert g is None
        elif name in want and not (name == "gate" and kd["gate"] is None):
            _near(g, *want[name], f"d{name}")
        else:
            assert g is None, name
    return got


WIDTHS = [1, 2, 3, 4, 5, 31, 32, 33, 63, 64, 99, 128, 129, 255, 256, 258, 511, 512, 777, 1024, 1025, 2048, 2051,
          4096, 4097, 8191, 8192]


@pytest.mark.parametrize("F", WIDTHS)
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_every_width(dg, device, F, kind):
    """Both directions at every width class, its borders and ragged widths; the number of rows is
    no multiple of a workgroup's."""
    for n, gate in ((1, "none"), (7, "col"), (67, "full")):
        c = _case(device, n, F, kind=kind, gate=gate)
        _check_forward(dg, *c)
        _check_backward(dg, *c)


@pytest.mark.parametrize("act,stream", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("gate,sigmoid", [("none", False), ("col", False), ("row", False), ("full", False),
                                          ("col", True), ("row", True), ("full", True)])
def test_types_and_gates(dg, device, act, stream, gate, sigmoid):
    for F in (3, 47, 128, 600, 2050):
        c = _case(device, 33, F, kind="layer", gate=gate, sigmoid=sigmoid, act=act, stream=stream)
        for half in (False, True):
            _check_forward(dg, *c, norm_bf16=half)
            _check_backward(dg, *c, grad_bf16=half)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("post,pre,block,vectors", [(False, True, True, True), (True, False, True, True),
                                                    (False, False, True, True), (False, True, False, True),
                                                    (True, True, True, False)])
def test_parts_left_out(dg, device, kind, post, pre, block, vectors):
    for F in (20, 300):
        c = _case(device, 41, F, kind=kind, post=post, pre=pre, block=block, vectors=vectors)
        _check_forward(dg, *c)
        _check_backward(dg, *c)


def test_no_gradient_of_the_stream_from_elsewhere(dg, device):
    dev, hst, kd, kh = _case(device, 50, 96, gate="col")
    dev["dRn"] = hst["dRn"] = None
    _check_backward(dg, dev, hst, kd, kh)


@pytest.mark.parametrize("n,F", [(20001, 99), (300000, 16), (4133, 256), (513, 4096)])
def test_many_rows(dg, device, n, F):
    """Column sums over more rows than one workgroup's step; the same bits twice."""
    c = _case(device, n, F, gate="col")
    a = _check_backward(dg, *c)
    b = dg.norm_residual_backward(c[0]["R"], c[0]["B"], c[0]["dZ"], c[0]["dRn"], **c[2])
    assert all(x is None or torch.equal(x, y) for x, y in zip(a, b))
    r1, r2 = _check_forward(dg, *c), dg.norm_residual(c[0]["R"], c[0]["B"], **c[2])
    assert torch.equal(r1[0], r2[0]) and torch.equal(r1[1], r2[1])


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("gate", ["col", "row", "full"])
def test_gradients_against_differences(dg, device, kind, gate):
    """L = <Z, dZ> + <Rn, dRn> in float64, differenced along random directions of every operand,
    against the device's gradients.  The step h = 1e-5 leaves h^2 of third derivatives (below
    1e-8 here) and 1e-11 / h of rounding; the device's share is 2^-17 of sum |g v|."""
    dev, hst, kd, kh = _case(device, 9, 24, kind=kind, gate=gate, sigmoid=True)
    # the gradients are taken at the stream after the block
    Rn, _ = ref.forward_stream(hst["R"], hst["B"], kh)
    dRn32 = torch.from_numpy(Rn.astype(np.float32)).to(device)
    got = dg.norm_residual_backward(dRn32, dev["B"], dev["dZ"], dev["dRn"], **kd)
    rng = np.random.default_rng(3)

    def L(ops, par):
        s, _ = ref.forward_stream(ops["R"], ops["B"], par)
        return (s * hst["dRn"]).sum() + (ref.forward_norm(s, par)[0] * hst["dZ"]).sum()

    for name in dg.NormGrads._fields:
        g = getattr(got, name)
        if g is None:
            continue
        g = g.double().cpu().numpy()
        where = hst if name in ("R", "B") else kh
        v = rng.standard_normal(g.shape)
        h = 1e-5
        side = []
        for sign in (1.0, -1.0):
            o, p = dict(hst), dict(kh)
            (o if where is hst else p)[name] = where[name] + sign * h * v
            side.append(L(o, p))
        want = (side[0] - side[1]) / (2 * h)
        assert abs((g * v).sum() - want) <= 1e-4 * np.abs(g * v).sum() + 1e-5, name


def test_rows_of_zeros_infinities_and_nan(dg, device):
    """A row's values reach no other row; a row of zeros is normed to its bias."""
    dev, hst, kd, kh = _case(device, 12, 130, kind="layer", gate="col")
    clean = dg.norm_residual(dev["R"], dev["B"], **kd)
    B = dev["B"].clone()
    B[3], B[5, 7], B[9, 0] = 0.0, float("nan"), float("inf")
    R = dev["R"].clone()
    R[11, 129] = float("-inf")
    Rn, Z = dg.norm_residual(R, B, **kd)
    keep = [0, 1, 2, 4, 6, 7, 8, 10]
    assert torch.equal(Rn[keep], clean[0][keep]) and torch.equal(Z[keep], clean[1][keep])
    want = R[3] + kd["scale"] * kd["gate"] * kd["post_bias"]
    assert torch.allclose(Rn[3], want, rtol=1e-6, atol=1e-6)
    assert torch.isnan(Rn[5]).all() and torch.isnan(Z[5]).all() and torch.isnan(Z[9]).all()
    assert torch.isnan(Z[11]).all() and Rn[11, 129] == float("-inf")
    zeros = torch.zeros(4, 64, device=device)
    _, Z = dg.norm_residual(zeros, kind="rms")
    assert torch.equal(Z, zeros)


def test_in_place_and_given_outputs(dg, device):
    dev, hst, kd, kh = _case(device, 70, 200, gate="full")
    want = dg.norm_residual(dev["R"], dev["B"], **kd)
    R = dev["R"].clone()
    Z = torch.full_like(R, float("nan"))
    Rn, Z2 = dg.norm_residual(R, dev["B"], Rn=R, Z=Z, **kd)
    assert Rn is R and Z2 is Z and torch.equal(R, want[0]) and torch.equal(Z, want[1])
    g = dg.norm_residual_backward(want[0], dev["B"], dev["dZ"], dev["dRn"], **kd)
    d = dev["dRn"].clone()
    g2 = dg.norm_residual_backward(want[0], dev["B"], dev["dZ"], d, dR=d, **kd)
    assert g2.R is d and all(x is None or torch.equal(x, y) for x, y in zip(g, g2))


def test_views_at_any_element(dg, device):
    """Rows that start at odd elements: a view into a larger buffer, and nothing behind it written."""
    for t in (torch.float32, torch.bfloat16):
        n, F = 21, 45
        flat = torch.randn(n * F + 9, device=device).to(t)
        R, B = flat[1:1 + n * F].view(n, F), torch.randn(n * F + 3, device=device).to(t)[3:].view(n, F)
        out = torch.full((n * F + 5,), 7.0, device=device, dtype=t)
        Rn, Z = dg.norm_residual(R, B, Rn=out[3:3 + n * F].view(n, F), norm_bf16=t == torch.bfloat16)
        want = dg.norm_residual(R.clone(), B.clone(), norm_bf16=t == torch.bfloat16)
        assert torch.equal(Rn, want[0]) and torch.equal(Z, want[1])
        assert (out[:3] == 7).all() and (out[3 + n * F:] == 7).all()


def test_another_stream_and_a_graph(dg, device):
    """A call on another stream, and the two directions captured together and replayed."""
    dev, hst, kd, kh = _case(device, 500, 128, gate="col")
    want = dg.norm_residual(dev["R"], dev["B"], **kd)
    back = dg.norm_residual_backward(want[0], dev["B"], dev["dZ"], dev["dRn"], **kd)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = dg.norm_residual(dev["R"], dev["B"], stream=side, **kd)
    got_back = dg.norm_residual_backward(got[0], dev["B"], dev["dZ"], dev["dRn"], stream=side, **kd)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert all(x is None or torch.equal(x, y) for x, y in zip(got_back, back))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    R = dev["R"].clone()
    with torch.cuda.graph(graph):
        cap = dg.norm_residual(R, dev["B"], **kd)
        cap_back = dg.norm_residual_backward(cap[0], dev["B"], dev["dZ"], dev["dRn"], **kd)
    for k in range(3):
        R.copy_(dev["R"] * (1.0 + 0.5 * k))
        eager = dg.norm_residual(R, dev["B"], **kd)
        eager_back = dg.norm_residual_backward(eager[0], dev["B"], dev["dZ"], dev["dRn"], **kd)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(cap[0], eager[0]) and torch.equal(cap[1], eager[1])
        assert all(x is None or torch.equal(x, y) for x, y in zip(cap_back, eager_back))


def test_more_than_2_to_the_31_elements(dg, device):
    """Offsets past 32 bits: the last rows of a bfloat16 stream of 2^31 + elements."""
    n, F = (1 << 24) + 3, 129
    R = torch.empty(n, F, device=device, dtype=torch.bfloat16)
    for a in range(0, n, 1 << 22):
        R[a:a + (1 << 22)].normal_()
    Z = torch.zeros_like(R)
    dg.norm_residual(R, pre_norm=True, norm_bf16=True, Z=Z)
    rows = torch.tensor([0, n // 2, n - 2, n - 1], device=device)
    want = dg.norm_residual(R[rows].contiguous(), norm_bf16=True)[1]
    assert torch.equal(Z[rows], want)


def test_refusals(dg, device):
    R = torch.randn(8, 32, device=device)
    B = torch.randn(8, 32, device=device)
    w = torch.ones(32, device=device)
    with pytest.raises(TypeError):
        dg.norm_residual(R.cpu())
    with pytest.raises(TypeError):
        dg.norm_residual(R.double())
    with pytest.raises(ValueError):
        dg.norm_residual(R.t())
    with pytest.raises(ValueError):
        dg.norm_residual(R, B[:4].contiguous())
    with pytest.raises(ValueError):
        dg.norm_residual(R, B, post_weight=w[:31].contiguous())
    with pytest.raises(ValueError):
        dg.norm_residual(R, gate=w)                              # a gate without a block
    with pytest.raises(ValueError):
        dg.norm_residual(R, pre_norm=False)
    with pytest.raises(ValueError):
        dg.norm_residual(R, B, kind="batch")
    for bad in (dict(eps=0.0), dict(eps=float("nan")), dict(eps=-1.0), dict(scale=float("nan")),
                dict(gate_sigmoid=True), dict(post_norm=False, post_weight=w), dict(Rn=B), dict(Z=R, Rn=R)):
        with pytest.raises(dg.DualGCNError) as e:
            dg.norm_residual(R, B, **bad)
        assert e.value.status == dg.ERR_INVALID_ARG
    with pytest.raises(dg.DualGCNError) as e:
        dg.norm_residual(torch.randn(2, 8193, device=device))
    assert e.value.status == dg.ERR_UNSUPPORTED
    with pytest.raises(dg.DualGCNError) as e:
        dg.norm_residual_backward(R, B, None, None)
    assert e.value.status == dg.ERR_INVALID_ARG
    with pytest.raises(dg.DualGCNError) as e:
        dg.norm_residual_backward(R, B, R.clone(), workspace=torch.empty(16, dtype=torch.uint8, device=device))
    assert e.value.status == dg.ERR_INVALID_ARG
