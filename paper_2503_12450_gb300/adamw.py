"""AdamW over named fp32 tensors, with the norm of all gradients, its clipping and averaged weights: two launches of
the library a step, and nothing that is copied to the host. A step whose gradients are not finite is skipped on the
device, and the count of steps stays there, so step() can be captured into a graph.
"""
import math

import torch

from . import lazymar as lm


class AdamW:
    """params and grads: dicts of fp32 (grads: or bf16) tensors of consecutive elements under the same names, which are
    updated where they are and have to stay there: their addresses are looked up once, which takes 65 us for 12 tensors and 1.5 ms
    for 384, more than a step of a small model. Matrices decay, vectors do not (`decays(name, tensor)` chooses otherwise).
    max_norm: gradients are scaled to this norm where theirs is larger. ema_decay: keeps averaged weights in `ema`.
    copies: dict of bf16 tensors that receive the weights after each step. lr may be changed between steps; a
    one-element fp32 tensor on the device is read by each step (under a captured graph too). One stream at a time."""

    def __init__(self, params, grads, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, max_norm=math.inf, ema_decay=None,
                 copies=None, decays=lambda name, tensor: tensor.dim() > 1):
        if set(params) != set(grads) or not params:
            raise lm.LazymarError(1, "params and grads: the same names, one at least")
        copies = copies or {}
        if not set(copies) <= set(params):
            raise lm.LazymarError(1, "copies: names of params required")
        self.lr, self.betas, self.eps, self.max_norm, self.ema_decay = lr, betas, eps, max_norm, ema_decay
        self.p, self.grads = dict(params), dict(grads)
        self.m = {k: torch.zeros_like(v) for k, v in params.items()}
        self.v = {k: torch.zeros_like(v) for k, v in params.items()}
        self.ema = {k: v.detach().clone() for k, v in params.items()} if ema_decay is not None else None
        # norm and factor (fp32), steps taken and skipped (int32)
        self.state = torch.zeros(4, device=next(iter(params.values())).device)
        self.list = lm.lazymar_params_create([dict(
            g=grads[k], p=v, m=self.m[k], v=self.v[k], ema=self.ema[k] if self.ema else None, copy=copies.get(k),
            weight_decay=weight_decay if decays(k, v) else 0.0) for k, v in params.items()])

    def step(self, scale=1.0):
        """scale: of the gradients, 1 / (loss scale, or number of batches accumulated)."""
        lm.lazymar_grad_norm(self.list, self.state, self.max_norm, scale)
        device = isinstance(self.lr, torch.Tensor)
        lm.lazymar_adamw(self.list, self.state, 0.0 if device else self.lr, self.betas[0], self.betas[1], self.eps,
                         0.0 if self.ema_decay is None else self.ema_decay, lr_device=self.lr if device else None)

    def clip(self, scale=1.0):
        """The norm and, in place, the clipped gradients (zeros where they are not finite), for a step made elsewhere."""
        lm.lazymar_grad_norm(self.list, self.state, self.max_norm, scale)
        lm.lazymar_clip_grads(self.list, self.state)

    def read(self):
        """(norm of the last step, its factor, steps, skipped steps); waits for the device."""
        whole = self.state.view(torch.int32).tolist()
        norm, factor = self.state[:2].tolist()
        return norm, factor, whole[2], whole[3]

    def state_dict(self):
        d = dict(m={k: v.clone() for k, v in self.m.items()}, v={k: v.clone() for k, v in self.v.items()}, state=self.state.clone())
        return dict(d, ema={k: v.clone() for k, v in self.ema.items()}) if self.ema else d

    def load_state_dict(self, d):
        """What state_dict() gave for the same tensors; nothing is changed where it does not fit."""
        mine = dict(m=self.m, v=self.v, **({"ema": self.ema} if self.ema else {}))
        if "state" not in d or d["state"].shape != self.state.shape or d["state"].dtype != self.state.dtype:
            raise lm.LazymarError(1, "state: four fp32 elements required")
        if self.ema and "ema" not in d:
            raise lm.LazymarError(1, "the state has no averaged weights")
        for name, tensors in mine.items():
            if set(d.get(name, ())) != set(tensors) or any(d[name][k].shape != t.shape for k, t in tensors.items()):
                raise lm.LazymarError(1, "the state's %s: tensors of these names and shapes required" % name)
        self.state.copy_(d["state"])
        for name, tensors in mine.items():
            for k, t in tensors.items():
                t.copy_(d[name][k])
