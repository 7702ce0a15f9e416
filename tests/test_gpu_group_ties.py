"""Group norms with ReLU on the GPU where elements are the mean of their group exactly: weight * u + bias is 0 there without a bias, and
nothing passes back.

The features are whole numbers, so that float64 holds their sums, their differences from any of them, and the mean where it is a whole
number too: there is nothing to be rounded, and the number of elements that pass is known from whole numbers alone."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dg(device):
    import paper_2609_01983_amd as dg
    return dg


def features(rng, sizes, F, G, offset):
    """int64 [n, F]: in every graph and group the mean is a whole number, and some elements (in three or more) have it."""
    out = []
    for rows in sizes:
        x = rng.integers(-40, 41, (rows, G, F // G))
        flat = x.transpose(1, 0, 2).reshape(G, -1)
        M = flat.shape[1]
        if M >= 3:
            mean = rng.integers(-3, 4, G)
            some = rng.choice(M, max(1, M // 8), replace=False)
            flat[:, some] = mean[:, None]
            rest = np.setdiff1d(np.arange(M), some)
            # what the sum is off goes to the others one by one
            off = M * mean - flat.sum(1)
            for g in range(G):
                flat[g, rest] += off[g] // rest.size
                flat[g, rest[:off[g] % rest.size]] += 1
            assert (flat.sum(1) == M * mean).all()
        out.append(flat.reshape(G, rows, F // G).transpose(1, 0, 2).reshape(rows, F) + offset)
    return np.concatenate(out)


# graphs for workgroups, for single wavefronts, long ones, and of few elements (the sizes are odd: a power of two divides exactly by itself)
SIZES = {"workgroups": [3, 5, 7, 11, 13, 49, 27, 99], "wavefronts": [1, 3, 5, 7, 9, 11, 49] * 310, "long": [9001, 3, 12345, 77], "few": [3, 1, 5, 7] * 40}


@pytest.mark.parametrize("offset", [0, 1000])
@pytest.mark.parametrize("F,G", [(1, 1), (3, 1), (12, 3), (9, 3), (64, 4), (99, 9), (100, 20), (300, 100), (520, 2)])
@pytest.mark.parametrize("sizes", SIZES)
def test_elements_that_are_the_mean(dg, device, sizes, F, G, offset):
    sizes = SIZES[sizes]
    rng = np.random.default_rng(F + offset)
    x = features(rng, sizes, F, G, offset)
    ptr = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    count = np.zeros(F)
    for lo, hi in zip(ptr[:-1], ptr[1:]):
        g = x[lo:hi].reshape(hi - lo, G, F // G)
        M = g.shape[0] * g.shape[2]
        count += (g * M > g.sum((0, 2))[None, :, None]).sum(0).reshape(F)
    for t in (torch.float32, torch.bfloat16) if offset == 0 else (torch.float32,):       # whole numbers up to 256 are bfloat16 numbers
        X = torch.from_numpy(x.astype(np.float32)).to(t).to(device)
        if not np.array_equal(X.double().cpu().numpy(), x):
            continue
        p = torch.from_numpy(ptr).to(device)
        par = dict(groups=G, bias=torch.zeros(F, device=device), act="relu")
        _, stats = dg.group_norm(X, p, **par)
        ones = torch.ones(X.shape, device=device)
        g = dg.group_norm_backward(X, ones, stats, p, **par)
        assert np.array_equal(g.bias.double().cpu().numpy(), count)
        mean = stats[..., 0].cpu().numpy()
        some = (np.diff(ptr) * (F // G) >= 3)
        assert (mean[some] == np.rint(mean[some])).all()
