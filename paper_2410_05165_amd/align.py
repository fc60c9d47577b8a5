"""Draft alignment training (AtSpeed-S, Sec. 3.1; AtSpeed-R, Sec. 3.2) of the
draft's item head, driven through atspeed_align_data / atspeed_align_step.

This module holds the buffers the two calls take (the batch, the fp32 master
copy of the head and the AdamW moments) and the learning-rate schedule (the
paper's implementation details: AdamW, lr 1e-3, cosine decay after a linear
warmup).  Every loss, gradient and update runs in the library's kernels.

A draft of the caller's own, trained by PyTorch, is aligned by distillation from
the target's top logits: ``distill`` is the loss with its gradient for autograd,
``atspeed_distill_loss`` and ``atspeed_distill_grad`` are the two calls under it.
"""
from __future__ import annotations

import functools
import math
from typing import Optional

from .binding import AlignArgs, Engine

MODES = {"S": 0, "R": 1}


def cosine_lr(step: int, total: int, peak: float, warmup: int) -> float:
    """Linear warmup to ``peak`` over ``warmup`` steps, then cosine decay to 0 at ``total``."""
    if warmup > 0 and step <= warmup:
        return peak * step / warmup
    if total <= warmup:
        return peak
    x = min(1.0, (step - warmup) / (total - warmup))
    return 0.5 * peak * (1.0 + math.cos(math.pi * x))


# Loaded by the first call: the schedule and the trainer come without PyTorch and _marshal.so.
@functools.lru_cache(maxsize=None)
def _calls():
    from .paged import _marshal, _run
    return _run, _marshal


def atspeed_distill_loss(logits, teacher_logit, teacher_index, tail=None, weight=None, temperature: float = 1.0,
                         reverse: bool = False):
    """The divergence of a draft's logits [rows, cols] (fp32 or bf16) from a teacher's top logits, a number a row.

    teacher_logit [rows, tops] of the logits' type at the columns teacher_index [rows, tops] (int32; outside the columns:
    no top); tail [rows] fp32: the log of the sum of exp(logit / temperature) over the teacher's other columns (None: it
    has none); weight [rows] fp32.  reverse: sum q log(q / p), which needs the tail, for sum p log(p / q).  Returns
    (loss [rows], saved), saved for atspeed_distill_grad.
    """
    run, calls = _calls()
    return run(calls.distill_loss, logits, logits, teacher_logit, teacher_index, tail, weight, temperature, reverse)


def atspeed_distill_grad(logits, teacher_index, saved, grad_loss=None, temperature: float = 1.0, out=None):
    """The gradient of atspeed_distill_loss with respect to the logits, in their type; grad_loss [rows] fp32 (None: 1)."""
    run, calls = _calls()
    return run(calls.distill_grad, logits, logits, teacher_index, saved, grad_loss, temperature, out)


@functools.lru_cache(maxsize=None)
def _autograd():
    import torch

    class Distill(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits, teacher_logit, teacher_index, tail, weight, temperature, reverse):
            loss, saved = atspeed_distill_loss(logits, teacher_logit, teacher_index, tail, weight, temperature, reverse)
            ctx.save_for_backward(logits, teacher_index, saved)
            ctx.temperature = temperature
            return loss

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, grad_loss):
            logits, teacher_index, saved = ctx.saved_tensors
            grad = atspeed_distill_grad(logits, teacher_index, saved, grad_loss.contiguous(), ctx.temperature)
            return grad, None, None, None, None, None, None

    return Distill


def distill(logits, teacher_logit, teacher_index, tail=None, weight=None, temperature: float = 1.0, reverse: bool = False):
    """atspeed_distill_loss for autograd: loss [rows] fp32, differentiable once and by the logits alone.

    A backward pass that is captured into a graph wants no other graph of the same parameters alive, as any other
    backward pass of PyTorch.
    """
    for name, t in (("teacher_logit", teacher_logit), ("tail", tail), ("weight", weight)):
        if t is not None and t.requires_grad:
            raise ValueError(f"{name}: no gradient flows to it; detach it")
    return _autograd().apply(logits, teacher_logit, teacher_index, tail, weight, temperature, reverse)


class AlignTrainer:
    """Buffers of one engine's draft-head training.

    ``mode``: "S" (strict verification's objective) or "R" (relaxed); ``alpha``
    the alignment strength (1: the alignment loss alone).  The master copy
    starts from the draft's current item head.
    """

    def __init__(self, eng: Engine, mode: str, alpha: float = 1.0, lr: float = 1e-3, betas=(0.9, 0.999),
                 eps: float = 1e-8, weight_decay: float = 0.01):
        torch = eng.torch
        if eng.draft_dev is None:
            raise ValueError("the engine has no draft model")
        self.eng = eng
        w = eng.w
        B, T, n = eng.cfg.max_batch, eng.max_nodes, eng.n_item
        dev = eng.device
        f32 = dict(dtype=torch.float32, device=dev)
        self.head = eng.draft_dev["lm_head_item"]            # the tensor the draft reads
        d = self.head.shape[1]
        self.ctx_weight = torch.zeros(B * T, **f32)
        self.label_weight = torch.zeros(B * T, **f32)
        self.root_weight = torch.zeros(B, **f32)
        self.log_pK = torch.zeros(B * w.L, **f32)
        self.lp_target = torch.zeros(B * T * n, **f32)
        self.root_target = torch.zeros(B * n, **f32)
        self.master = self.head.float().contiguous().clone()
        self.m = torch.zeros(n * d, **f32)
        self.v = torch.zeros(n * d, **f32)
        self.grad = torch.zeros(n * d, **f32)
        self.args = AlignArgs()
        a = self.args
        a.mode, a.alpha = MODES[mode], alpha
        a.ctx_weight, a.label_weight = self.ctx_weight.data_ptr(), self.label_weight.data_ptr()
        a.root_weight, a.log_pK = self.root_weight.data_ptr(), self.log_pK.data_ptr()
        a.lp_target, a.root_target = self.lp_target.data_ptr(), self.root_target.data_ptr()
        a.master, a.adam_m, a.adam_v, a.grad = (x.data_ptr() for x in (self.master, self.m, self.v, self.grad))
        a.hidden_out = None
        a.lr, a.beta1, a.beta2, a.eps, a.weight_decay = lr, betas[0], betas[1], eps, weight_decay
        a.step = 0

    def data(self, items, n_items, lens=None):
        """The batch of the engine's last prefill: items [B, S, L] int32, n_items [B],
        lens [B, S] (None: whole items) (device)."""
        self.eng.atspeed_align_data(items, lens, n_items, self.args)

    def step(self, lr: Optional[float] = None, hidden_out=None) -> float:
        """One AdamW step; returns the loss before it."""
        a = self.args
        a.step += 1
        if lr is not None:
            a.lr = lr
        a.hidden_out = None if hidden_out is None else hidden_out.data_ptr()
        return self.eng.atspeed_align_step(a)
