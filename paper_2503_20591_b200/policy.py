"""Learned placement policies in PyTorch: the library's policy operators with autograd.

A policy scores every host for every request, logits [..., H], -inf where the host cannot take it.
`distill_loss` trains it on the hosts nbos_place_batch chose, `balance_loss` keeps it from sending everything
to few hosts, `sample_hosts` lets it answer. Every step runs in the library's CUDA kernels.
"""
from __future__ import annotations

import torch

from . import binding


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, hosts, teacher_logits, temperature):
        rows = logits.shape[:-1]
        loss = torch.empty(rows, dtype=torch.float32, device=logits.device)
        stats = torch.empty((*rows, 2), dtype=torch.float32, device=logits.device)
        binding.nbos_policy_distill(logits, hosts, teacher_logits, loss, stats, temperature=temperature)
        ctx.save_for_backward(logits, hosts, teacher_logits, stats)
        ctx.temperature = temperature
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_loss):
        logits, hosts, teacher_logits, stats = ctx.saved_tensors
        grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        binding.nbos_policy_distill_backward(logits, hosts, teacher_logits, stats, grad,
                                             grad_loss=grad_loss.float().contiguous(), temperature=ctx.temperature)
        return grad, None, None, None


class _BalanceLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, hosts):
        groups = logits.shape[:-2]
        loss = torch.empty(groups, dtype=torch.float32, device=logits.device)
        counts = torch.empty((*groups, logits.shape[-1]), dtype=torch.int32, device=logits.device)
        shares = torch.empty(counts.shape, dtype=torch.float32, device=logits.device)
        stats = torch.empty((*logits.shape[:-1], 2), dtype=torch.float32, device=logits.device)
        binding.nbos_policy_balance(logits, hosts, loss, counts, shares, stats)
        ctx.save_for_backward(logits, hosts, stats)
        ctx.mark_non_differentiable(counts, shares)
        return loss, counts, shares

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_loss, _counts, _shares):
        logits, hosts, stats = ctx.saved_tensors
        grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        binding.nbos_policy_balance_backward(logits, hosts, stats, grad, grad_loss=grad_loss.float().contiguous())
        return grad, None


def distill_loss(logits, hosts, teacher_logits=None, temperature: float = 1.0) -> torch.Tensor:
    """Loss per row [...] of logits [..., H] against the teacher's hosts [..., k] (int32, -1 = none; what
    nbos_place_batch writes can be passed as it is) with logits [..., k], [k] or None (all equal). The gradient is that of
    `logits`; the teacher has none."""
    if torch.is_grad_enabled() and isinstance(teacher_logits, torch.Tensor) and teacher_logits.requires_grad:
        raise ValueError("teacher_logits has no gradient here: detach it")
    return _DistillLoss.apply(logits, hosts, teacher_logits, float(temperature))


def balance_loss(logits, hosts):
    """(loss [N], counts [N, H], mean shares [N, H]) of logits [N, B, H] and the hosts that the policy chose
    [N, B, k] (sample_hosts, or its best ones: its own load is what the loss evens out); without the leading N for logits
    [B, H]. The loss has a gradient, counts and shares have none."""
    if logits.dim() > 3:
        raise ValueError("logits must be [N, B, H] or [B, H]")
    return _BalanceLoss.apply(logits, hosts)


def sample_hosts(logits, uniforms, temperature=None, top_k=None, top_p=None, min_p=None):
    """(hosts [..., draws], found [...]): distinct hosts drawn with the given random numbers [..., draws], one
    setting per row or one number for all."""
    rows = logits.shape[:-1]

    def per_row(v, dtype):
        if v is None or isinstance(v, torch.Tensor):
            return v
        return torch.full(rows, v, dtype=dtype, device=logits.device)

    hosts = torch.empty(uniforms.shape, dtype=torch.int32, device=logits.device)
    found = torch.empty(rows, dtype=torch.int32, device=logits.device)
    binding.nbos_policy_sample(logits, uniforms, hosts, found, temperature=per_row(temperature, torch.float32),
                               top_k=per_row(top_k, torch.int32), top_p=per_row(top_p, torch.float32),
                               min_p=per_row(min_p, torch.float32))
    return hosts, found
