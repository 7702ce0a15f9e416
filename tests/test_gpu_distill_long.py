"""Long rows of the distillation loss that are not split: their sums of exponentials, whose terms are
equal (every rounding of such a sum is alike, so a long chain of additions shows), and of random logits.  Bounds
as in distillref.py."""
import numpy as np
import pytest
import torch

import distillref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dg(device):
    import paper_2609_01983_amd as dg
    return dg


# more than 128 rows: a workgroup sweeps a row by itself; 128: four share it
@pytest.mark.parametrize("n", [130, 128])
@pytest.mark.parametrize("y", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1.0, 2.0])
def test_equal_terms(dg, device, n, y, T):
    C = (1 << 20) - 1
    level = -T * (0.25 + torch.arange(n, device=device) / 64.0)     # a value a row: how roundings add up goes by it
    # one class in eight has the row's largest logit, in runs, so that whoever sums some of a row meets it early
    top = torch.arange(C, device=device) % 16384 < 2048
    Y = torch.where(top, 0.0, level[:, None]).to(y)
    tops = int(top.sum())
    ids = torch.tensor([[5, C - 1]], dtype=torch.int32, device=device).repeat(n, 1)
    teacher = torch.tensor([[1.0, 0.5]], device=device).repeat(n, 1)
    labels = torch.full((n,), 7, dtype=torch.int32, device=device)
    G, loss = dg.distill_xent(Y, ids, teacher, labels, temperature=T, soft_scale=0.5, hard_scale=0.25)
    h = lambda t: t.cpu().numpy()  # noqa: E731
    for v in range(n):
        z = float(Y[v, 2048])
        q = [np.exp(z / t) / (tops + (C - tops) * np.exp(z / t)) for t in (T, 1.0)]
        want = 0.5 * T * q[0] + 0.25 * q[1]              # a class that neither the teacher nor the label takes
        bound = ref.U * want * (ref.K + 6 * abs(z)) + 2 * ref.U * want
        got = G[v, [2048, 16383, 500000]].double().cpu().numpy()
        assert (np.abs(got - want) <= bound).all(), (v, np.abs(got / want - 1).max() / ref.U)
    one = ref.distill(h(Y[:1].double()), h(ids[:1]), h(teacher[:1]).astype(np.float64), h(labels[:1]), T, 0.5, 0.25)
    assert (np.abs(G[0].double().cpu().numpy() - one[0][0]) <= one[2][0] + 2 * ref.U * np.abs(one[0][0])).all()
    assert torch.isfinite(loss).all()


def test_random_logits(dg, device):
    n, C, K = 131, 300001, 9
    g = torch.Generator(device=device).manual_seed(4)
    Y = (torch.randn(n, C, device=device, generator=g) * 3).to(torch.bfloat16)
    ids = torch.randint(0, C, (n, K), device=device, generator=g).to(torch.int32)
    teacher = torch.randn(n, K, device=device, generator=g)
    labels = torch.randint(-1, C, (n,), device=device, generator=g).to(torch.int32)
    for T in (1.0, 2.5):
        G, loss = dg.distill_xent(Y, ids, teacher, labels, temperature=T, soft_scale=1.0 / 128, hard_scale=1.0 / 128)
        h = lambda t: t.cpu().numpy()  # noqa: E731
        wG, wl, bG, bl = ref.distill(Y.double().cpu().numpy(), h(ids), h(teacher).astype(np.float64), h(labels), T, 1.0 / 128, 1.0 / 128)
        assert (np.abs(h(G.double()) - wG) <= bG + 2 * ref.U * np.abs(wG)).all()
        assert (np.abs(h(loss.double()) - wl) <= bl).all()
