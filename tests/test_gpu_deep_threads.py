"""Calls of the deep-GCN operators from several host threads at once, each on a stream of its own: every
thread finishes all its calls, with the bits of a call by itself.  An exception in a thread is the test's."""
from concurrent.futures import ThreadPoolExecutor

import pytest
import torch

pytestmark = pytest.mark.gpu

CALLS = 20


@pytest.fixture(scope="module")
def dg(device):
    import paper_2609_01983_amd as dg
    return dg


def test_threads_on_streams_of_their_own(dg, device):
    g = torch.Generator(device=device).manual_seed(2)
    make = lambda *s: torch.randn(*s, device=device, generator=g)  # noqa: E731
    n, F = 3001, 96
    R, B, dZ, w = make(n, F), make(n, F), make(n, F), make(F)
    ids = torch.randint(0, F, (n, 6), device=device, generator=g).to(torch.int32)
    teacher = make(n, 6)
    W8 = dg.quantize_weight_fp8(make(F, 40))
    works = [lambda: dg.norm_residual(R, B, post_weight=w, gate=w, gate_sigmoid=True),
             lambda: [x for x in dg.norm_residual_backward(R, B, dZ, None, post_weight=w, gate=w, gate_sigmoid=True)
                      if x is not None],
             lambda: dg.distill_xent(R, ids, teacher, temperature=2.0, soft_scale=0.1),
             lambda: dg.distill_xent(R, ids, teacher, temperature=20.0, soft_scale=0.1),
             lambda: (dg.update_fp8(*dg.quantize_fp8(B), *W8),)]
    wants = [f() for f in works]
    torch.cuda.synchronize()

    def run(k):
        stream = torch.cuda.Stream(device)
        done = 0
        with torch.cuda.stream(stream):
            for _ in range(CALLS):
                got = works[k]()
                assert len(got) == len(wants[k]) and all(torch.equal(x, y) for x, y in zip(got, wants[k])), k
                done += 1
            stream.synchronize()
        return done

    with ThreadPoolExecutor(10) as pool:
        for f in [pool.submit(run, k % 5) for k in range(10)]:
            assert f.result(timeout=60) == CALLS
