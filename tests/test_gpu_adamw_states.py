"""AdamW steps whose states or surroundings are not the ordinary ones: captured steps, gradients that are not finite, 8-bit states
that follow a gradient far slower than a code's step.  References and tolerances as in test_gpu_adamw.py."""
import math

import pytest
import torch

import policy_reference as ref
from paper_2512_23353_amd import isopo
from paper_2512_23353_amd.policy import PolicyLinear, PolicyTrainer

pytestmark = pytest.mark.gpu


def test_a_captured_step_says_that_it_repeats(gpu_device):
    layer = PolicyLinear(16, 8, dtype=torch.float32, device=gpu_device)
    layer.weight_grad = torch.ones(8, 16, device=gpu_device)
    trainer = PolicyTrainer([layer])
    opt = isopo.AdamW([torch.zeros(64, device=gpu_device)])
    g = [torch.ones(64, device=gpu_device)]
    opt.step(g, 1e-2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.warns(UserWarning, match="repeats step 2"):
            opt.step(g, 1e-2)
        with pytest.raises(RuntimeError, match="captured"):
            trainer.step()
    for k in range(3):                                # m after one real step and k + 1 replays: the formula's, whatever the step's number
        graph.replay()
        torch.cuda.synchronize()
        want = 1 - 0.9 ** (k + 2)
        assert bool(((opt.m[0] - want).abs() <= 2.0 ** -20).all())
    trainer.step()
    assert trainer.optimiser.steps_done == 1 and layer.weight_grad is None
