"""Group norms on the GPU where single wavefronts take the graphs (from 2,048 on, short on the average) and where one long
graph's elements are past 2^31, against float64 (bounds: groupref.py).

A row of F features takes 1, 8, 16, 32 or 64 lanes of a wavefront (up to 3, 32, 64, 128 and more features); groups are whole quads of
features in a power of two of lanes, or not.  Every width has float32 and bfloat16 on either side, and
a batch with some graphs past what a wavefront takes."""
import numpy as np
import pytest
import torch

import groupref

pytestmark = pytest.mark.gpu

EPS = 1e-5


@pytest.fixture(scope="module")
def dg(device):
    import paper_2609_01983_amd as dg
    return dg


def host(t):
    return t.double().cpu().numpy()


def near(got, want, bound, what):
    bound = bound + (groupref.BF16 * (np.abs(want) + bound) if got.dtype == torch.bfloat16 else groupref.U * np.abs(want)) + 1e-44
    bad = ~(np.abs(host(got) - want) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} outside, first at {np.argwhere(bad)[0]}: {host(got)[bad][:3]} for {want[bad][:3]}"


def batch(lanes):
    """Sizes of 2,500 graphs whose rows take at most 16 turns of a wavefront on the average, 64 / lanes rows a turn."""
    rng = np.random.default_rng(lanes)
    mean = 1024 // lanes
    sizes = np.minimum(rng.integers(0, 61, 2500), rng.integers(0, 2 * min(mean, 30) + 1, 2500))
    turns = 64 // lanes                              # past a wavefront's 32 turns, backward 8, and some of its exact size
    sizes[rng.choice(2500, 6, replace=False)] = [33 * turns, 32 * turns, 32 * turns + 1, 8 * turns, 8 * turns + 1, 70 * turns]
    return sizes


def lanes_of(F, G):
    D = F // G
    width = 256 if D > 256 else min(F, 256 // D * D)
    return 1 if width < 4 else 8 if width <= 32 else 16 if width <= 64 else 32 if width <= 128 else 64


@pytest.mark.parametrize("types", ["float32", "bfloat16", "bfloat16 in", "bfloat16 out"])
@pytest.mark.parametrize("F,G", [(1, 1), (2, 1), (3, 3), (20, 4), (32, 2), (60, 5), (64, 8), (99, 9), (128, 8), (128, 1), (200, 40), (256, 32),
                                 (300, 3), (520, 8)])
def test_one_wavefront_for_each_graph(dg, device, F, G, types):
    lanes = lanes_of(F, G)
    sizes = batch(lanes)
    ptr = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32) + 3
    n = int(ptr[-1]) + 2                             # rows of no graph before and behind
    assert n // len(sizes) * lanes <= 1024
    rng = np.random.default_rng(F)
    to = lambda a: torch.from_numpy(a.astype(np.float32)).to(device)  # noqa: E731
    act = ("relu", "silu", None)[F % 3]
    x_bf, y_bf = types in ("bfloat16", "bfloat16 in"), types in ("bfloat16", "bfloat16 out")
    X = to(rng.standard_normal((n, F)) * np.exp(0.5 * rng.standard_normal(F)) + 0.5 * rng.standard_normal(F))
    dY = to(rng.standard_normal((n, F)))
    X, dY = X.to(torch.bfloat16) if x_bf else X, dY.to(torch.bfloat16) if y_bf else dY
    w, b, p = to(1 + 0.3 * rng.standard_normal(F)), to(0.3 * rng.standard_normal(F)), torch.from_numpy(ptr).to(device)
    par = dict(groups=G, weight=w, bias=b, act=act)
    Y, stats = dg.group_norm(X, p, eps=EPS, out_bf16=y_bf, **par)
    want, bound, st, rows = groupref.forward(host(X), ptr, G, host(w), host(b), act, EPS)
    near(Y, want, bound, "Y")
    assert (Y[~rows] == 0).all()
    got, spread = host(stats), 1.0 / st[..., 1]
    assert (np.abs(got[..., 0] - st[..., 0]) <= 1e-11 * (spread + np.abs(st[..., 0]))).all()
    assert (np.abs(got[..., 1] / st[..., 1] - 1) <= 1e-11).all()
    g = dg.group_norm_backward(X, dY, stats, p, **par)
    for one, wants, name in zip(g, groupref.backward(host(X), host(dY), ptr, G, host(w), host(b), act, EPS), ("dX", "dweight", "dbias")):
        near(one, *wants, name)
    assert (g.X[~rows] == 0).all()


def test_long_graphs_past_2_to_the_31_elements(dg, device):
    """Two graphs of 2^23 rows and more, of which the second has the 2^31st element.  Their statistics against float64 sums over blocks of rows;
    Y, and dX for a dY that is not Y, in rows around the first, the 2^31st element's, the last and tiles' ends, by the
    formulas with the sums of all rows; the vectors' gradients over all rows.

    Statistics and sums: 1e-11 as elsewhere for the first; the vectors' gradients and dX's means sum 2^23 rows of d and d u, each off by
    groupref's bound of their magnitudes.  Y is within 8 2^-24 M, M = |u w| + |b|, and a half bfloat16 step; dX within 32 2^-24 of its terms, and a half step."""
    n, F, G = (1 << 24) + 77, 136, 8
    g = torch.Generator(device=device).manual_seed(2)
    X = torch.empty(n, F, device=device, dtype=torch.bfloat16).normal_(generator=g)
    dY = torch.empty(n, F, device=device, dtype=torch.bfloat16).normal_(generator=g)
    X[1 << 23:] += 3.0
    ptr = [0, 1 << 23, n - 40]
    p = torch.tensor(ptr, device=device, dtype=torch.int32)
    w, b = 1 + 0.3 * torch.randn(F, device=device, generator=g), 0.3 * torch.randn(F, device=device, generator=g)
    par = dict(groups=G, weight=w, bias=b, act="relu")
    Y, stats = dg.group_norm(X, p, eps=EPS, out_bf16=True, **par)
    grads = dg.group_norm_backward(X, dY, stats, p, **par)
    D, U, W, Bv = F // G, groupref.U, w.double(), b.double()
    dw, db, Mw, Mb = (torch.zeros(F, device=device, dtype=torch.float64) for _ in range(4))
    wide = lambda v: v.repeat_interleave(D)  # noqa: E731
    groups = lambda v: v.view(G, D).sum(1)  # noqa: E731
    step = 1 << 18
    for k in range(2):
        lo, hi = ptr[k], ptr[k + 1]
        M = (hi - lo) * D
        blocks = [slice(r, min(hi, r + step)) for r in range(lo, hi, step)]
        mean = groups(sum(X[r].double().sum(0) for r in blocks)) / M
        v = groups(sum((X[r].double() - wide(mean)).square().sum(0) for r in blocks)) / M
        r_ = 1.0 / torch.sqrt(v + EPS)
        assert ((stats[k, :, 0] - mean).abs() <= 1e-11 * (1 / r_ + mean.abs())).all() and ((stats[k, :, 1] / r_ - 1).abs() <= 1e-11).all()
        mf, rf = wide(mean), wide(r_)

        def parts(rows):
            u = (X[rows].double() - mf) * rf
            return u, torch.where(u * W + Bv > 0, dY[rows].double(), 0.0)

        s1, s2, m1, m2 = (torch.zeros(F, device=device, dtype=torch.float64) for _ in range(4))
        for rows in blocks:
            u, d = parts(rows)
            s1, s2 = s1 + d.sum(0), s2 + (d * u).sum(0)
            m1, m2 = m1 + d.abs().sum(0), m2 + (d * u).abs().sum(0)
        dw, db, Mw, Mb = dw + s2, db + s1, Mw + m2, Mb + m1
        t1, t2 = wide(groups(s1 * W)) / M, wide(groups(s2 * W)) / M
        e1, e2 = wide(groups(m1 * W.abs())) / M, wide(groups(m2 * W.abs())) / M
        at = {lo, lo + 1, hi - 2, hi - 1, (lo + hi) // 2}
        at |= {q for c in (1 << 31, 1 << 30, 1 << 32) for q in (c // F - 1, c // F, c // F + 1)}
        at |= {q for t in range(16300, 16500) for q in (lo + t, hi - t)}
        rows = torch.tensor(sorted(q for q in at if lo <= q < hi), device=device)
        u, d = parts(rows)
        pre = u * W + Bv
        want = torch.where(pre > 0, pre, 0.0)
        bound = 8 * U * ((u * W).abs() + Bv.abs())
        assert ((Y[rows].double() - want).abs() <= bound + 2.0 ** -8 * (want.abs() + bound)).all(), k
        want = rf * (d * W - t1 - u * t2)
        bound = 32 * U * rf * ((d * W).abs() + e1 + u.abs() * e2)
        assert ((grads.X[rows].double() - want).abs() <= bound + 2.0 ** -8 * (want.abs() + bound)).all(), k
    for got, want, size in ((grads.weight, dw, Mw), (grads.bias, db, Mb)):
        assert ((got.double() - want).abs() <= 32 * U * size + U * want.abs()).all()
    assert (Y[ptr[2]:] == 0).all() and (grads.X[ptr[2]:] == 0).all()
