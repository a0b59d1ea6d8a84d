"""Activations and their slopes at the ends of the types: finite where the formulas are, with no infinity times zero on the way."""
import pytest
import torch

import policy_reference as ref
from paper_2512_23353_amd import isopo

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("act", ref.ACTS[1:])
def test_slopes_far_from_zero(gpu_device, dtype, act):
    """From |z| = 30 on slopes are 0 and 1 to 20 digits, so Delta is dY or nothing; and Y is Z or nothing."""
    t = ref.DTYPES[dtype]
    ends = torch.tensor([30.0, 1e3, 1e9, 1.5e13, 1e19, 2e19, 1e20, 1e30, 3e38], device=gpu_device).to(t)
    z = torch.cat([ends, -ends]).repeat(8)[None].contiguous()            # [1, 144]
    dy = torch.randn(z.shape, device=gpu_device).to(t)
    W = torch.zeros((144, 8), dtype=t, device=gpu_device)
    delta, _, db = isopo.linear_backward(dy, W, z, act, need_db=True)
    want = torch.where(z > 0, dy, torch.zeros_like(dy))
    assert torch.allclose(delta, want, rtol=0, atol=1e-6) and torch.allclose(db, want[0].float(), rtol=0, atol=1e-6)
    assert torch.equal(delta[z > 0], dy[z > 0])
    # forward: z as the bias of a sum of nothing
    y, kept = isopo.linear(torch.zeros((1, 8), dtype=t, device=gpu_device), W, bias=z[0].contiguous(), act=act, keep_z=True)
    assert torch.equal(kept, z) and torch.allclose(y, torch.where(z > 0, z, torch.zeros_like(z)), rtol=0, atol=1e-6)
