"""What a residual block leaves, from its operands R and B, for every pair of types.

Z norms the stream as it is stored.  Beside a float32 Z a bfloat16 stream Rn is the formula's sum rounded to
float32 and then to bfloat16 (to nearest even), so it is known to the bit from float64: a stream that is off by one
step somewhere moves that element of Z by up to 2^-7 of itself, far over a float32 Z's bound.
Elements that an error of EDGE of the sum's magnitudes could round to another bfloat16 number are not decided by
float64 either, nor is their rows' Z: they have to be few (sums that cancel to nothing, one in 10,000 of R + 0.7 B)."""
import numpy as np
import pytest
import torch

import normref as ref

pytestmark = pytest.mark.gpu

# float64 sums of a row in chains of at most 64, some stages on: 2^-53 of the magnitudes each
EDGE = 2.0 ** -45
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def dg(device):
    import paper_2609_01983_amd as dg
    return dg


def to_bf16(x):
    """Float64 numbers rounded to float32 and then to bfloat16, both to nearest even."""
    m, e = np.frexp(x.astype(np.float32).astype(np.float64))
    return np.ldexp(np.rint(m * 256.0), e - 8)


def through_norm(x, err, p):
    """How far errors of a row's elements of at most `err` move its norm: the derivative's bound."""
    layer = p["kind"] == "layer"
    u, rho, _ = ref.unit(x, layer, p["eps"])
    mean = lambda a: a.mean(1, keepdims=True)  # noqa: E731
    w = np.abs(ref.one(p["pre_weight"], x.shape[1]))
    return 1.01 * w * rho * (err + (mean(err) if layer else 0.0) + np.abs(u) * mean(err * np.abs(u)))


def case(device, n, F, act, stream, kind="rms", post=True, gate="none", sigmoid=False, seed=0):
    rng = np.random.default_rng(seed + 8209 * n + F)

    def make(a, t):
        d = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(TYPES[t])
        return d.to(device), d.double().numpy()

    R, hR = make(rng.standard_normal((n, F)) * np.exp(0.5 * rng.standard_normal((n, 1))) + 0.1, stream)
    B, hB = make(rng.standard_normal((n, F)) * np.exp(0.5 * rng.standard_normal((n, 1))) + 0.2, act)
    layer = kind == "layer"
    kd = dict(post_norm=post, gate_sigmoid=sigmoid, scale=0.7, kind=kind, eps=1e-5)
    kh = dict(kd)
    for name, there, about in (("post_weight", post, 1.0), ("post_bias", post and layer, 0.0),
                               ("pre_weight", True, 1.0), ("pre_bias", layer, 0.0)):
        kd[name], kh[name] = make(about + 0.2 * rng.standard_normal(F), "f32") if there else (None, None)
    shape = {"none": None, "col": (F,), "row": (n, 1), "full": (n, F)}[gate]
    kd["gate"], kh["gate"] = (None, None) if shape is None else make(0.5 + 0.5 * rng.standard_normal(shape),
                                                                    act if gate == "full" else "f32")
    return (R, B, kd), (hR, hB, kh)


def check(dg, dev, hst, stream, z):
    (R, B, kd), (hR, hB, kh) = dev, hst
    Rn, Z = dg.norm_residual(R, B, norm_bf16=z == "bf16", **kd)
    want, bound = ref.forward_stream(hR, hB, kh)
    got, gz = Rn.double().cpu().numpy(), Z.double().cpu().numpy()
    rows, err = np.ones(len(want), dtype=bool), np.zeros_like(want)
    if stream == "f32":
        err = bound + ref.U * np.abs(want)
        assert (np.abs(got - want) <= err).all()
    elif z == "f32":
        edge = bound / (ref.K * ref.U) * EDGE            # bound is K u of the sum's magnitudes
        sure = to_bf16(want - edge) == to_bf16(want + edge)
        rows = sure.all(1)
        want = to_bf16(want)
        assert sure.mean() > 0.999 and rows.mean() > 0.5
        off = (got != want) & sure
        assert not off.any(), f"{off.sum()} of {off.size} of the stream are not the sum, rounded"
    else:
        assert (np.abs(got - want) <= bound + ref.BF16 * (np.abs(want) + bound)).all()
        want = got
    wz, bz = ref.forward_norm(want, kh)
    bz = bz + through_norm(want, err, kh)
    bz = bz + (ref.BF16 * (np.abs(wz) + bz) if z == "bf16" else ref.U * np.abs(wz))
    bad = ~(np.abs(gz - wz) <= bz)[rows]
    assert not bad.any(), f"{bad.sum()} of {bad.size} of Z outside"


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("stream", ["f32", "bf16"])
@pytest.mark.parametrize("z", ["f32", "bf16"])
def test_every_pair_of_types(dg, device, act, stream, z):
    for n, F in ((60000, 3), (5001, 47), (3000, 128), (1001, 400)):
        for kind in ("rms", "layer"):
            check(dg, *case(device, n, F, act, stream, kind=kind, gate="col"), stream, z)


@pytest.mark.parametrize("F", [1, 2, 4, 31, 64, 99, 160, 192, 256, 300, 512, 700, 1000, 1500, 2048, 2500, 4096, 5000, 8191])
def test_every_width_of_a_bfloat16_stream(dg, device, F):
    n = 300000 // F + 1
    check(dg, *case(device, n, F, "f32", "bf16"), "bf16", "f32")
    check(dg, *case(device, n, F, "bf16", "bf16", kind="layer"), "bf16", "f32")


@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("gate,sigmoid", [("none", False), ("col", True), ("row", False), ("row", True), ("full", False),
                                          ("full", True)])
def test_gates_of_a_bfloat16_stream(dg, device, gate, sigmoid, post):
    for act in ("f32", "bf16"):
        for F in (2, 130, 600):
            check(dg, *case(device, 200000 // F, F, act, "bf16", post=post, gate=gate, sigmoid=sigmoid), "bf16", "f32")


@pytest.mark.parametrize("scale", [0.7, 0.5, 0.1, 1.0, -0.3, 1.0 / 3.0, 1e-3])
def test_sums_in_the_middle(dg, device, scale):
    """R + scale B of bfloat16 operands, with many sums in the middle of two bfloat16 numbers but for float64's
    rounding (0.7: where B is a multiple of 5)."""
    (R, B, kd), (hR, hB, kh) = case(device, 3001, 128, "bf16", "bf16", post=False)
    kd["scale"] = kh["scale"] = scale
    sums = hR + scale * hB
    assert (to_bf16(sums * (1 - 2.0 ** -20)) != to_bf16(sums * (1 + 2.0 ** -20))).mean() > 5e-4
    check(dg, (R, B, kd), (hR, hB, kh), "bf16", "f32")


def test_a_bfloat16_stream_that_is_not_finite(dg, device):
    """Infinities and NaN stay in their rows, in their places for RMS norms; a sum past bfloat16's largest is
    an infinity; large and small rows are as the formula has them."""
    (R, B, kd), (hR, hB, kh) = case(device, 40, 200, "f32", "bf16")
    clean, _ = dg.norm_residual(R, B, **kd)
    R, B = R.clone(), B.clone()
    B[3, 7], B[5, 0], R[7, 199] = float("nan"), float("inf"), float("-inf")
    top = torch.finfo(torch.bfloat16).max
    R[9], B[9] = top, 1.0
    B[11] *= 1e30                                        # squares past float32's largest
    B[13] *= 1e-30
    Rn, Z = dg.norm_residual(R, B, **kd)
    keep = [v for v in range(40) if v not in (3, 5, 7, 9, 11, 13)]
    assert torch.equal(Rn[keep], clean[keep])
    assert torch.isnan(Rn[3]).all() and torch.isnan(Z[3]).all()
    assert torch.isnan(Rn[5, 0]) and torch.equal(Rn[5, 1:], R[5, 1:])
    assert Rn[7, 199] == float("-inf") and torch.equal(Rn[7, :199], clean[7, :199])
    assert torch.equal(Rn[9], R[9])                      # less than half a step more
    want = to_bf16(ref.forward_stream(hR, B.double().cpu().numpy(), kh)[0])
    assert np.array_equal(Rn[[11, 13]].double().cpu().numpy(), want[[11, 13]])
    Rn, _ = dg.norm_residual(R[9:10].contiguous(), torch.full_like(B[:1], 1e38), post_norm=False, scale=10.0)
    assert torch.isinf(Rn).all()
