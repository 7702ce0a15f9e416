"""Gates of blocks with one feature, where a gate for each node has the shape of a gate for each element."""
import pytest
import torch

import normref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dg(device):
    import paper_2609_01983_amd as dg
    return dg


@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gate_type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("grad_bf16", [False, True])
def test_one_feature(dg, device, act, gate_type, grad_bf16):
    n = 333
    g = torch.Generator(device=device).manual_seed(1)
    R = torch.randn(n, 1, device=device, generator=g)
    B = torch.randn(n, 1, device=device, generator=g).to(act)
    gate = torch.randn(n, 1, device=device, generator=g).to(gate_type)
    block = dict(post_norm=False, gate=gate, scale=0.5, pre_norm=False)
    if gate_type is torch.bfloat16 and act is torch.float32:
        with pytest.raises(TypeError):                   # neither kind of gate
            dg.norm_residual(R, B, **block)
        return
    Rn, _ = dg.norm_residual(R, B, **block)
    h = lambda t: t.double().cpu().numpy()  # noqa: E731
    want = h(R) + 0.5 * h(gate) * h(B)
    assert (abs(h(Rn) - want) <= 4 * ref.U * (abs(h(R)) + abs(0.5 * h(gate) * h(B)))).all()
    d = torch.randn(n, 1, device=device, generator=g)
    got = dg.norm_residual_backward(Rn, B, None, d, grad_bf16=grad_bf16, **block)
    # in B's type the gate is one for each element, whose gradient has the gradients' type
    full = gate_type is act
    assert got.gate.dtype is (torch.bfloat16 if full and grad_bf16 else torch.float32)
    want = 0.5 * h(d) * h(B)
    near = 4 * ref.U + (ref.BF16 if got.gate.dtype is torch.bfloat16 else 0.0)
    assert got.gate.shape == (n, 1) and (abs(h(got.gate) - want) <= near * abs(want)).all()
