"""Group norms on the GPU with a workspace of exactly the bytes that they ask for, between bytes that stay as they were; results
against float64 (bounds: groupref.py)."""
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


def near(got, want, bound, what):
    g = got.double().cpu().numpy()
    bad = ~(np.abs(g - want) <= bound + groupref.U * np.abs(want) + 1e-44)
    assert not bad.any(), f"{what}: {bad.sum()} outside, first at {np.argwhere(bad)[0]}"


def guarded(device, size):
    buf = torch.full((size + 1024,), 0x5A, dtype=torch.uint8, device=device)
    return buf, buf[512:512 + size]


# long graphs from the first row of all, from inside tiles, side by side, over several tiles, one after many short ones
@pytest.mark.parametrize("sizes", [[5000], [1, 5000, 1], [300, 4000, 300, 300, 4000], [1500, 1500, 1500, 1500], [9000, 0, 0, 3000, 77],
                                   [1] * 5000 + [4000] + [0] * 3000 + [2000], [31, 33] * 1500 + [7000], [256] * 30 + [257] * 30])
@pytest.mark.parametrize("F,G", [(96, 4), (128, 128), (20, 5), (600, 2), (400, 2)])
def test_exact_workspaces(dg, device, sizes, F, G):
    ptr = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    n, B = int(ptr[-1]), len(sizes)
    rng = np.random.default_rng(n + F)
    to = lambda a: torch.from_numpy(a.astype(np.float32)).to(device)  # noqa: E731
    X, dY = to(rng.standard_normal((n, F)) + 0.5 * rng.standard_normal(F)), to(rng.standard_normal((n, F)))
    w, b, p = to(1 + 0.3 * rng.standard_normal(F)), to(0.3 * rng.standard_normal(F)), torch.from_numpy(ptr).to(device)
    par = dict(groups=G, weight=w, bias=b, act="relu")
    host = [t.double().cpu().numpy() for t in (X, dY, w, b)]
    buf, ws = guarded(device, dg.group_norm_workspace_bytes(n, F, G, B))
    Y, stats = dg.group_norm(X, p, eps=EPS, workspace=ws if ws.numel() else None, **par)
    assert (buf[:512] == 0x5A).all() and (buf[-512:] == 0x5A).all()
    want, bound, _, _ = groupref.forward(host[0], ptr, G, host[2], host[3], "relu", EPS)
    near(Y, want, bound, "Y")
    buf, ws = guarded(device, dg.group_norm_workspace_bytes(n, F, G, B, backward=True))
    g = dg.group_norm_backward(X, dY, stats, p, workspace=ws, **par)
    assert (buf[:512] == 0x5A).all() and (buf[-512:] == 0x5A).all()
    for one, wants, name in zip(g, groupref.backward(host[0], host[1], ptr, G, host[2], host[3], "relu", EPS), ("dX", "dweight", "dbias")):
        near(one, *wants, name)
