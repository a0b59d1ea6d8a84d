"""The policy's layers where autograd, the training loop or the module's owner does what it may: gradients and inputs of any strides, no
gradient at all, parameters written from outside, microbatches one after the other.  Against torch's own layers in fp32, with the
tolerance of test_gpu_policy.py."""
import pytest
import torch
from torch import nn

from paper_2512_23353_amd import isopo
from paper_2512_23353_amd.policy import IsopoUpdate, PolicyLinear, PolicyTrainer, token_logprob

pytestmark = pytest.mark.gpu


def _rel(a, b):
    a, b = a.detach().double(), b.detach().double()
    return float((a - b).norm() / b.norm())


def _leaf(t):
    return t.detach().clone().requires_grad_()


@pytest.mark.parametrize("act", ("none", "silu"))
def test_gradients_of_any_strides(gpu_device, act):
    """Behind the layer: a concatenation (its gradient's rows start anywhere), a slice, a transpose, a broadcast sum.  Before it: sliced inputs and
    residuals."""
    torch.manual_seed(0)
    layer = PolicyLinear(12, 20, bias=True, act=act, dtype=torch.float32, device=gpu_device)
    layer.bias.data.normal_()
    f = {"none": lambda z: z, "silu": nn.functional.silu}[act]
    wide, rest, side = torch.randn(9, 31, device=gpu_device), torch.randn(9, 27, device=gpu_device), torch.randn(9, 3, device=gpu_device)
    c = torch.randn(9, 23, device=gpu_device)
    behind = (lambda y: (torch.cat([side, y], dim=1) * c).sum(), lambda y: (torch.cat([y, side], dim=1) * c).sum(), lambda y: (y[:, 3:] * c[:, :17]).sum(),
              lambda y: (y.t() * c[:, :20].t()).sum(), lambda y: y.sum(), lambda y: (y[::2] * c[::2, :20]).sum(), lambda y: y[4:5].sum())
    for k in (0, 1, 5, 19):
        for loss in behind:
            x, r = _leaf(wide), _leaf(rest)
            w, b = _leaf(layer.weight), _leaf(layer.bias)
            layer.weight_grad = layer.bias_grad = None
            y = layer(x[:, k:k + 12], residual=r[:, k % 8:k % 8 + 20])
            loss(y).backward()
            x2, r2 = _leaf(wide), _leaf(rest)
            y2 = f(nn.functional.linear(x2[:, k:k + 12], w, b)) + r2[:, k % 8:k % 8 + 20]
            loss(y2).backward()
            for got, want in ((y, y2), (x.grad, x2.grad), (r.grad, r2.grad), (layer.weight_grad, w.grad), (layer.bias_grad, b.grad)):
                assert _rel(got, want) < 1e-5
    x = torch.randn(12, 9, device=gpu_device)
    assert _rel(layer(x.t()), f(nn.functional.linear(x.t(), layer.weight, layer.bias))) < 1e-5
    x = torch.randn(1, 12, device=gpu_device).expand(6, 12)
    assert _rel(layer(x), f(nn.functional.linear(x, layer.weight, layer.bias))) < 1e-5


def test_logits_of_any_strides(gpu_device):
    z = torch.randn(50, 9, device=gpu_device)
    y = torch.randint(0, 50, (9,), device=gpu_device, dtype=torch.int32)
    for view in (lambda t: t.t(), lambda t: t[:, :1].t().expand(9, 50)):
        a, b = _leaf(z), _leaf(z)
        w = torch.arange(1.0, 10.0, device=gpu_device)
        (token_logprob(view(a), y) * w).sum().backward()
        (torch.log_softmax(view(b), dim=1).gather(1, y.long()[:, None])[:, 0] * w).sum().backward()
        assert _rel(a.grad, b.grad) < 1e-5


def test_a_loaded_checkpoint_stays_loaded(gpu_device):
    """bf16 layers with fp32 masters: a step of learning rate 0 leaves what was loaded, and one moves from there."""
    torch.manual_seed(2)
    layer = PolicyLinear(64, 32, device=gpu_device)
    trainer = PolicyTrainer([layer], weight_decay=0.0)
    other = torch.randn(32, 64, device=gpu_device).bfloat16()
    for load in (lambda: layer.load_state_dict({"weight": other}), lambda: setattr(layer, "weight", nn.Parameter(other.clone())),
                 lambda: setattr(layer.weight, "data", other.clone()), lambda: (layer.weight.data.copy_(other), trainer.read_parameters())):
        layer.weight_grad = torch.randn(32, 64, device=gpu_device)
        trainer.step(lr=0.1)
        new = (layer.weight != other).detach()
        assert new.float().mean() > 0.9
        load()
        layer.weight_grad = torch.randn(32, 64, device=gpu_device)
        trainer.step(lr=0.0)
        assert torch.equal(layer.weight, other) and torch.equal(trainer.optimiser.masters[0][new], other.float()[new])
