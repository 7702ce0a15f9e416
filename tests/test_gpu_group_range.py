"""Group norms of features that lie further apart than float32 reaches, on the GPU against float64 (bounds: groupref.py).

Such features are numbers like others: a group of +a and -a has the normed features +1 and -1 also where 2 a or the variance is
past float32's range, and its gradient is divided by a spread of up to 3.4e38.  The bounds are groupref's, and half a
step of the smallest numbers of an output's type: 2^-150, bfloat16 2^-134 (a whole float32 step is left for both types)."""
import numpy as np
import pytest
import torch

import groupref

pytestmark = pytest.mark.gpu

EPS = 1e-5
TOP = float(np.finfo(np.float32).max)


@pytest.fixture(scope="module")
def dg(device):
    import paper_2609_01983_amd as dg
    return dg


def host(t):
    return t.double().cpu().numpy()


def near(got, want, bound, what):
    bf16 = got.dtype == torch.bfloat16
    bound = bound + (2.0 ** -8 * (np.abs(want) + bound) + 2.0 ** -134 if bf16 else 2.0 ** -24 * np.abs(want)) + 2.0 ** -149
    bad = ~(np.abs(host(got) - want) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} outside, first at {np.argwhere(bad)[0]}: {host(got)[bad][:3]} for {want[bad][:3]}"


def sizes_to_ptr(sizes):
    return np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)


# graphs taken by workgroups, by single wavefronts (many graphs), over tiles (one long graph), by the float64 branch of few elements
SIZES = {"workgroups": [40, 1, 0, 33, 64, 100], "wavefronts": [3, 9, 0, 1, 12] * 500, "tiles": None, "few": [1, 2, 3, 4] * 30}


def far(rng, n, F, G, kind):
    """Features of both signs at float32's end; in every second group ordinary ones."""
    x = rng.standard_normal((n, F))
    if kind == "ends":
        big = np.where(rng.random((n, F)) < 0.5, TOP, -TOP) * (1 - 0.2 * rng.random((n, F)))
    elif kind == "one far":                          # one element of a group far from the others
        big = np.full((n, F), -TOP) * (1 - 1e-3 * rng.random((n, F)))
        big[rng.integers(0, n, max(1, n // 50))] *= -1.0
    else:                                            # spreads from 1 up to the end, a power of two a row
        big = np.ldexp(x, rng.integers(90, 126, (n, 1)))
    wide = np.repeat(np.arange(G) % 2 == 0, F // G)
    return np.where(wide, big, x).astype(np.float32)


@pytest.mark.parametrize("act", ["relu", "silu"])
@pytest.mark.parametrize("kind", ["ends", "one far", "spread"])
@pytest.mark.parametrize("F,G", [(2, 2), (64, 8), (99, 9), (300, 300), (520, 2)])
@pytest.mark.parametrize("sizes", SIZES)
def test_features_at_the_ends_of_float32(dg, device, sizes, F, G, kind, act):
    ptr = sizes_to_ptr(SIZES[sizes] or ([9000, 7, 11000] if F < 64 else [1500, 7, 2600]))
    n = int(ptr[-1])
    rng = np.random.default_rng(n + F)
    to = lambda a: torch.from_numpy(a).to(device)  # noqa: E731
    x = far(rng, n, F, G, kind)
    w, b = (1 + 0.3 * rng.standard_normal(F)).astype(np.float32), (0.3 * rng.standard_normal(F)).astype(np.float32)
    p = to(ptr)
    for bf16 in (False, True):
        t = torch.bfloat16 if bf16 else torch.float32
        X = torch.clamp(to(x), -3e38, 3e38).to(t)
        par = dict(groups=G, weight=to(w), bias=to(b), act=act)
        Y, stats = dg.group_norm(X, p, eps=EPS, out_bf16=bf16, **par)
        want, bound, st, _ = groupref.forward(host(X), ptr, G, w.astype(float), b.astype(float), act, EPS)
        got = host(stats)
        assert (np.abs(got[..., 0] - st[..., 0]) <= 1e-11 * (1.0 / st[..., 1] + np.abs(st[..., 0]))).all()
        assert (np.abs(got[..., 1] / st[..., 1] - 1) <= 1e-11).all()
        near(Y, want, bound, "Y")
        for size in (1.0, 1e30):
            dY = to((size * rng.standard_normal((n, F))).astype(np.float32)).to(t)
            g = dg.group_norm_backward(X, dY, stats, p, **par)
            wants = groupref.backward(host(X), host(dY), ptr, G, w.astype(float), b.astype(float), act, EPS)
            for one, other, name in zip(g, wants, ("dX", "dweight", "dbias")):
                near(one, *other, f"{name} for dY of {size}")


def test_one_graph_of_two_values(dg, device):
    """+a and -a: u is +1 and -1 to the last place, whatever a is."""
    for a in (1e19, 2.0 ** 99, 2.0 ** 100, 2.0 ** 101, 1e38, 1.7e38, 1.8e38, TOP):
        for n, F in ((2, 1), (6, 8), (30000, 16)):
            X = torch.full((n, F), a, device=device)
            X[::2] = -a
            Y, stats = dg.group_norm(X, groups=1)
            want = torch.ones(n, F, device=device)
            want[::2] = -1.0
            assert (Y - want).abs().max() <= 2.0 ** -22, a


def test_subnormal_features_keep_their_places(dg, device):
    """Features of a few of float32's smallest steps beside a spread of nothing: u = (X - m) / sqrt(eps), to float32's roundings.
    Half of m as two numbers is off by 2^-150 at most, as the second is a multiple of 2^-149; half of X less the first is rounded to such
    a multiple too: X - m is off by 2 (2^-150 + 2^-150) = 2^-148 at most, and u by r 2^-148."""
    for n, F, G in ((64, 8, 2), (20000, 8, 2)):
        rng = np.random.default_rng(n)
        X = torch.from_numpy(np.ldexp(rng.integers(-40, 41, (n, F)).astype(np.float64), -149).astype(np.float32)).to(device)
        for eps in (1e-5, 2.0 ** -126):
            Y, _ = dg.group_norm(X, groups=G, eps=eps)
            want, bound, st, _ = groupref.forward(host(X), None, G, None, None, None, eps)
            near(Y, want, bound + np.repeat(st[0, :, 1], F // G) * 2.0 ** -148, "Y")
