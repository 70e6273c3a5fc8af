"""Clipping of lists whose tensors have different types, into outputs off their boundary (needs a
GPU).  A block's warps go from piece to piece by themselves, so that one is at a tensor of 16 bits
while another is at one of 32: what they keep in shared memory must not overlap."""
import random

import pytest
import torch

from paper_2205_11048_gb300 import binding as B
from tests.test_gpu_worker import NORM_BOUND, TINY, TYPES, U, UNIT, exact_norm, gen, gradients, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("types", [TYPES, TYPES[::-1], [torch.float32] + [torch.bfloat16] * 3, [torch.float16, torch.float32]],
                         ids=["all", "reversed", "few of 32 bits", "alternating"])
@pytest.mark.parametrize("parts,most", [(40, 200_000), (700, 5000), (700, 20_000), (1200, 9000), (2500, 3000)])
def test_lists_of_different_types(types, parts, most):
    w = B.Worker()
    for seed in range(4):
        r = random.Random(seed + parts)
        sizes = [int(most ** r.random()) + r.randrange(most // 4) for _ in range(parts)]
        grads = gradients(gen(seed), sizes, types, seed)
        want = exact_norm(grads)
        limit = 0.5 * want
        outs = [[torch.full((t.numel() + 3,), 7.0, dtype=dtype or t.dtype, device="cuda")[1 + i % 3:][:t.numel()]
                 for i, t in enumerate(grads)] for dtype in (torch.float32, None, torch.bfloat16)]
        for out in outs:
            norm = w.clip_grads(B.grad_parts(grads, out), limit)
            assert abs(float(norm) - want) <= NORM_BOUND * want
        w.sync()
        # all parts at once: the list is long
        exact = torch.cat([t.double() for t in grads]) * min(1.0, limit / (want + 1e-6))
        tol = (NORM_BOUND + 4 * U) * exact.abs()
        for out in outs:
            unit = torch.cat([torch.full((t.numel(),), UNIT[t.dtype] if t.dtype != torch.float32 else 0.0, device="cuda") for t in out])
            within(torch.cat([t.double() for t in out]), exact, tol * 1.01 + unit * exact.abs() + TINY[torch.float16], "clipped")
    w.close()
