"""A policy's layers, objective and optimiser step around the ISOPO layer step, as torch.autograd sees them.

    up = PolicyLinear(hidden, ffn, act="gelu")          # forward, and Delta, dX, db in backward, in the library's kernels
    logp = token_logprob(logits, targets)               # differentiable, with the entropy if wanted
    update = IsopoUpdate([up, ...], variant="interacting", lam=1e-3)
    trainer = PolicyTrainer([up, ...], lr=1e-3, state_bits=8)

    update.begin(seq_offsets, advantages)               # the microbatch's sequences
    logp.sum().backward()                               # no advantages: the hook listings' objective
    trainer.step()                                      # AdamW over all layers' gradients, few launches

A layer's weight gradient is formed where its backward pass has X and Delta: the ISOPO gradient of the layer step while an IsopoUpdate
is in force, else the plain Delta^T X.  It is kept in fp32 beside the parameter (`weight_grad`, `bias_grad`), as the library's calls
return it, and accumulates until the trainer's step.  No arithmetic of the method happens here.
"""
from __future__ import annotations

import math
from typing import Iterable, Optional

import numpy as np
import torch
from torch import nn
from torch.autograd.function import once_differentiable

from . import isopo
from .hooks import VARIANTS, _hip_layer_step


def _rows(t: torch.Tensor) -> torch.Tensor:
    """t [n, d] as isopo.linear takes rows (contiguous, 16 bytes aligned, apart by whole vectors), or a copy that is: gradients of slices,
    concatenations and broadcasts come as they may."""
    vec = 16 // t.element_size()
    apart = t.stride(0)
    if (t.shape[1] > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and (apart < t.shape[1] or apart % vec or apart >= 1 << 22)) or t.data_ptr() % 16:
        return t.clone(memory_format=torch.contiguous_format)
    return t


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, layer, recorded):
        # (needs_input_grad is the tensors' own, whether autograd records or not)
        keep_z = layer.act != "none" and recorded and any(ctx.needs_input_grad)
        out = isopo.linear(x, weight, bias, layer.act, residual, keep_z=keep_z)
        y, z = out if keep_z else (out, None)
        ctx.layer, ctx.has_bias, ctx.has_residual = layer, bias is not None, residual is not None
        mark = getattr(layer.update, "mark", None)
        ctx.mark = mark and mark()
        ctx.save_for_backward(x, weight, z)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, z = ctx.saved_tensors
        dy = _rows(dy)
        delta, dx, db = isopo.linear_backward(dy, weight, z, ctx.layer.act, need_dx=ctx.needs_input_grad[0],
                                              need_db=ctx.has_bias and ctx.needs_input_grad[2])
        if ctx.needs_input_grad[1]:
            ctx.layer.add_weight_grad(x, delta, ctx.mark)
        if db is not None:
            ctx.layer.bias_grad = db if ctx.layer.bias_grad is None else ctx.layer.bias_grad + db
        return dx, None, None, dy if ctx.has_residual else None, None, None


class PolicyLinear(nn.Module):
    """act(x W^T + bias) + residual for x [..., d_in], a linear layer of the policy (isopo.linear).  d_in and d_out are multiples of 8 (bf16)
    or 4 (fp32), as the layer step asks; a vocabulary of another size is padded to one.  After a backward pass
    `weight_grad` [d_out, d_in] and `bias_grad` [d_out] hold the gradients in fp32; the parameters' .grad stay as they are."""

    def __init__(self, d_in: int, d_out: int, bias: bool = False, act: str = "none", dtype=torch.bfloat16, device=None):
        super().__init__()
        if act not in isopo._ACTS:
            raise ValueError(f"act must be one of {tuple(isopo._ACTS)}")
        self.act = act
        self.weight = nn.Parameter(torch.empty((d_out, d_in), dtype=dtype, device=device))
        self.bias = nn.Parameter(torch.zeros(d_out, dtype=dtype, device=device)) if bias else None
        nn.init.normal_(self.weight, std=1.0 / math.sqrt(d_in))
        self.update = None                  # (layer, X, Delta) -> dW, or an IsopoUpdate; None: Delta^T X
        self.weight_grad: Optional[torch.Tensor] = None
        self.bias_grad: Optional[torch.Tensor] = None

    def add_weight_grad(self, x: torch.Tensor, delta: torch.Tensor, mark: Optional[int] = None) -> None:
        x, delta = x.contiguous(), delta.contiguous()
        if self.update is not None:
            dw = self.update(self, x, delta) if mark is None else self.update(self, x, delta, mark)
        else:
            dw = isopo.weighted_grad(isopo.Layer(x, delta, [0, x.shape[0]]), None)
        if self.weight_grad is None:
            self.weight_grad = dw
        else:
            self.weight_grad += dw

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        rows = _rows(x.reshape(-1, x.shape[-1]))
        if residual is not None:
            residual = _rows(residual.reshape(-1, residual.shape[-1]))
        y = _Linear.apply(rows, self.weight, self.bias, residual, self, torch.is_grad_enabled())
        return y.reshape(*x.shape[:-1], y.shape[-1])


class _TokenLogprob(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, inv_temperature, entropy):
        out = isopo.token_logprob(logits, targets, inv_temperature, entropy=entropy)
        ctx.save_for_backward(logits, targets, out["lse"], out.get("entropy"))
        ctx.inv_temperature = inv_temperature
        if entropy:
            return out["logp"], out["entropy"]
        return out["logp"]

    @staticmethod
    @once_differentiable
    def backward(ctx, g, h=None):
        logits, targets, lse, ent = ctx.saved_tensors
        d = isopo.token_logprob_backward(logits, targets, lse, g.contiguous(), ctx.inv_temperature, entropy=ent,
                                         grad_entropy=None if ent is None else h.contiguous())
        return d, None, None, None


def token_logprob(logits: torch.Tensor, targets: torch.Tensor, inv_temperature: float = 1.0, entropy: bool = False):
    """log-probabilities [n] (fp32) of the targets (int32 [n], negative: padding) under softmax(inv_temperature * logits), logits
    [n, vocab]; with `entropy` also the entropies [n].  Differentiable in the logits."""
    if logits.stride(-1) != 1 or logits.stride(0) < logits.shape[1]:
        logits = logits.contiguous()
    return _TokenLogprob.apply(logits, targets, float(inv_temperature), bool(entropy))


class IsopoUpdate:
    """While in force, the weight gradient of every given PolicyLinear is the ISOPO gradient of its microbatch (the same layer steps
    and options as hooks.IsopoHooks).  Layers with a bias are refused: the method says nothing of one."""

    def __init__(self, layers: Iterable[PolicyLinear], variant: str = "interacting", lam: float = 1e-3, relative_reg: bool = True,
                 n_samples: int = 32, pqr=(0.0, -1.0, -2.0), reg3=(0.0, 0.0, 0.0), seed: int = 0, ema_decay: float = 0.9):
        if variant not in VARIANTS:
            raise ValueError(f"variant must be one of {VARIANTS}")
        self.layers = list(layers)
        if any(layer.bias is not None for layer in self.layers):
            raise ValueError("an ISOPO layer has no bias")
        self.cfg = {"variant": variant, "lam": float(lam), "relative_reg": bool(relative_reg), "n_samples": int(n_samples),
                    "pqr": tuple(pqr), "reg3": tuple(reg3), "generator": torch.Generator(device="cpu").manual_seed(seed),
                    "ema_decay": float(ema_decay)}
        self._ema = {}
        self._offsets = self._advantages = None
        self._begun, self._used = 0, False          # calls of begin(); whether a backward pass has been of the last one's sequences
        for layer in self.layers:
            layer.update = self

    def begin(self, seq_offsets, advantages: torch.Tensor) -> None:
        """The next backward passes are of these sequences: row offsets (host) and one fp32 advantage each (device).  To be called before or after
        the microbatch's forward pass; what runs forward once a backward pass has been of these sequences is another microbatch, which
        needs its own."""
        self._offsets = np.ascontiguousarray(np.asarray(seq_offsets, dtype=np.int32))
        self._advantages = advantages
        self._begun, self._used = self._begun + 1, False

    def mark(self) -> int:
        """The earliest call of begin() that a backward pass of what runs forward now can be of."""
        return self._begun + self._used

    def __call__(self, layer, x, delta, mark: Optional[int] = None):
        """dW of a layer's X and Delta; mark: what mark() said at its forward pass."""
        if self._offsets is None or (mark is not None and self._begun < mark):
            raise RuntimeError("begin() tells which sequences a backward pass is of")
        if int(self._offsets[-1]) != x.shape[0]:
            raise ValueError(f"seq_offsets cover {int(self._offsets[-1])} tokens, the layer saw {x.shape[0]}")
        cfg = self.cfg
        if cfg["variant"] == "interacting_ema":
            if layer not in self._ema:
                self._ema[layer] = torch.zeros(2, dtype=torch.float32, device=x.device)
            cfg = dict(cfg, ema_state=self._ema[layer])
        dw = _hip_layer_step(x, delta, self._offsets, self._advantages, cfg)
        self._used = True
        return dw

    def remove(self) -> None:
        for layer in self.layers:
            layer.update = None


class PolicyTrainer:
    """AdamW on the layers' weights (and biases).  bf16 parameters get fp32 master copies.  The policy's objective is to be
    maximised: the step goes along the gradients.

    The parameters are the layers' at each step.  Where one was written or replaced since the last (a checkpoint loaded into it, other
    storage or another Parameter), its master takes over what changed.  Writes through `.data` leave no trace on a parameter:
    read_parameters() after them."""

    def __init__(self, layers: Iterable[PolicyLinear], lr: float = 1e-4, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.0,
                 state_bits: int = 32, max_norm: Optional[float] = 1.0):
        self.layers = list(layers)
        self.lr, self.max_norm = float(lr), max_norm
        self._slots = [(layer, "weight") for layer in self.layers] + [(layer, "bias") for layer in self.layers if layer.bias is not None]
        params = self._params()
        self._masters = [p.detach().float() for p in params] if params[0].dtype == torch.bfloat16 else None
        self.optimiser = isopo.AdamW(params, masters=self._masters, state_bits=state_bits, betas=betas, eps=eps, weight_decay=weight_decay,
                                     maximize=True)
        self._seen = self._written(params)

    def _params(self) -> list:
        return [getattr(layer, name) for layer, name in self._slots]

    @staticmethod
    def _written(params) -> list:
        """What differs where a parameter has been written or has other storage."""
        return [(p.data_ptr(), p._version) for p in params]

    def _follow(self, every: bool = False) -> list:
        params = self.optimiser.params[:] = self._params()
        self.optimiser.find_params()
        now = self._written(params)
        if self._masters is not None:
            for p, master, seen, at in zip(params, self._masters, self._seen, now):
                if every or seen != at:
                    p, master = p.detach().reshape(-1), master.view(-1)
                    master.copy_(torch.where(p == master.to(p.dtype), master, p.float()))        # what was not changed keeps its low bits
        self._seen = now
        return params

    def read_parameters(self) -> None:
        """The masters take over the parameters' values where these are not their rounded copies."""
        self._follow(every=True)

    def step(self, lr: Optional[float] = None) -> Optional[torch.Tensor]:
        """One step along the gradients gathered since the last; returns their norm (device) if it is limited.  Not for a graph to capture:
        replays would repeat this one step."""
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("an optimiser step cannot be captured: replays would repeat it with its number, lr and rounding")
        grads = [getattr(layer, name + "_grad") for layer, name in self._slots]
        if any(g is None for g in grads):
            raise RuntimeError("a layer has no gradient: was it part of the backward pass?")
        params = self._follow()
        norm = self.optimiser.step(grads, self.lr if lr is None else float(lr), max_norm=self.max_norm)
        # the library writes behind autograd's back: a backward pass of what ran forward with the old weights is refused, as after torch's own steps
        torch.autograd.graph.increment_version(params)
        self._seen = self._written(params)
        for layer, name in self._slots:
            setattr(layer, name + "_grad", None)
        return norm
