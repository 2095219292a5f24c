"""Learned placement policies in PyTorch: the library's policy operators with autograd.

A policy scores every host for every request, logits [..., H], -inf where the host cannot take it.
`distill_loss` trains it on the hosts nbos_place_batch chose, `balance_loss` keeps it from sending everything
to few hosts, `sample_hosts` lets it answer. A policy of two towers, whose score is a product of two vectors, is trained by
`tower_distill_loss` without its table of logits; `block_norm` is what stands between two residual blocks of a tower,
`clip_gradients` bounds the step. Every step runs in the library's CUDA kernels.
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


def _empty_like(t):
    return torch.empty_like(t, memory_format=torch.contiguous_format)   # 3 us less than torch.empty from its parts


class _TowerDistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, requests, host_vectors, hosts, teacher_logits, temperature, asks, room, gradient_values):
        rows = requests.shape[:-1]
        loss = torch.empty(rows, dtype=torch.float32, device=requests.device)
        stats = torch.empty((*rows, 2 + hosts.shape[-1]), dtype=torch.float32, device=requests.device)
        binding.nbos_policy_towers(requests, host_vectors, hosts, teacher_logits, loss, stats, temperature=temperature, asks=asks, room=room)
        ctx.save_for_backward(requests, host_vectors, hosts, teacher_logits, asks, room, stats)
        ctx.temperature, ctx.gradient_values = temperature, gradient_values
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_loss):
        requests, host_vectors, hosts, teacher_logits, asks, room, stats = ctx.saved_tensors
        grads = [_empty_like(t) if need else None for t, need in zip((requests, host_vectors), ctx.needs_input_grad)]
        binding.nbos_policy_towers_backward(requests, host_vectors, hosts, teacher_logits, stats, *grads,
                                            grad_loss=grad_loss.float().contiguous(), temperature=ctx.temperature, asks=asks, room=room,
                                            gradient_values=ctx.gradient_values)
        return (*grads, None, None, None, None, None, None)


class _BlockNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, residual, branch, gate, post_weight, pre_weight, residual_scale, eps):
        ctx.set_materialize_grads(False)
        out, normed = _empty_like(residual), _empty_like(residual)
        stats = torch.empty((*residual.shape[:-1], 2), dtype=torch.float32, device=residual.device)
        binding.nbos_policy_block_norm(residual, branch, gate, post_weight, pre_weight, out, normed, stats, residual_scale, eps)
        ctx.save_for_backward(residual, branch, gate, post_weight, pre_weight, stats)
        ctx.residual_scale = residual_scale
        return out, normed

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_out, grad_normed):
        *inputs, stats = ctx.saved_tensors
        grads = [_empty_like(t) if need else None for t, need in zip(inputs, ctx.needs_input_grad)]
        if grad_out is None and grad_normed is None:
            return (*(None if g is None else g.zero_() for g in grads), None, None)
        rows_alike = [None if g is None else g.contiguous() for g in (grad_out, grad_normed)]
        binding.nbos_policy_block_norm_backward(*inputs, stats, *rows_alike, *grads, residual_scale=ctx.residual_scale)
        return (*grads, None, None)


def distill_loss(logits, hosts, teacher_logits=None, temperature: float = 1.0) -> torch.Tensor:
    """Loss per row [...] of logits [..., H] against the teacher's hosts [..., k] (int32, -1 = none; what
    nbos_place_batch writes can be passed as it is) with logits [..., k], [k] or None (all equal). The gradient is that of
    `logits`; the teacher has none."""
    if torch.is_grad_enabled() and isinstance(teacher_logits, torch.Tensor) and teacher_logits.requires_grad:
        raise ValueError("teacher_logits has no gradient here: detach it")
    return _DistillLoss.apply(logits, hosts, teacher_logits, float(temperature))


def tower_distill_loss(requests, host_vectors, hosts, teacher_logits=None, temperature: float = 1.0, asks=None, room=None,
                       gradient_values: int = 2) -> torch.Tensor:
    """distill_loss of a two-tower policy's logits, requests [N, B, D] times host_vectors [N, H, D] (or without N; bfloat16 or
    float16), -inf where the request's asks [N, B, 4] exceed the host's room [N, H, 4] (int32; None: all fit). The table of
    logits [N, B, H] is never stored; of its gradient the backward pass holds pieces of about 512 MB at a time. gradient_values = 1 rounds
    that gradient to the vectors' type before it is multiplied, for up to 1.8 times the speed; 2 keeps what the rounding takes off."""
    if gradient_values not in (1, 2):
        raise ValueError("gradient_values must be 1 or 2")
    if torch.is_grad_enabled() and isinstance(teacher_logits, torch.Tensor) and teacher_logits.requires_grad:
        raise ValueError("teacher_logits has no gradient here: detach it")
    return _TowerDistillLoss.apply(requests, host_vectors, hosts, teacher_logits, float(temperature), asks, room, gradient_values)


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


def block_norm(residual, branch, gate=None, post_weight=None, pre_weight=None, residual_scale: float = 1.0, eps: float = 1e-6):
    """(r, h) with r = residual_scale * residual + gate * norm(branch) * post_weight, the stream behind a residual block, and
    h = norm(r) * pre_weight, what the next block reads; norm(v) = v / sqrt(mean(v^2) + eps) over the last dimension. residual, branch
    [..., D]; gate like them, [N, 1, D] beside [N, B, D], or [D]; weights [D]."""
    return _BlockNorm.apply(residual, branch, gate, post_weight, pre_weight, float(residual_scale), float(eps))


def clip_gradients(parameters, max_norm: float, norm_type: float = 2.0) -> torch.Tensor:
    """Scales the gradients of `parameters` in place by min(1, max_norm / (norm + 1e-6)), norm their global 2-norm (or, norm_type
    inf, their largest magnitude), and returns the norm, a scalar on the device. Parameters without a gradient are passed
    over, one that is given twice counts once. Nothing waits for the device."""
    kinds = {2.0: binding.NBOS_NORM_2, float("inf"): binding.NBOS_NORM_INF}
    if norm_type not in kinds:
        raise ValueError("norm_type must be 2 or inf")
    parameters = [parameters] if isinstance(parameters, torch.Tensor) else list(parameters)
    found = list(dict.fromkeys(p.grad for p in parameters if p.grad is not None))   # (tensors hash by identity)
    grads = [g if g.is_contiguous() else g.contiguous() for g in found]
    device = grads[0].device if grads else parameters[0].device if parameters else "cuda"
    norm = torch.empty((), dtype=torch.float32, device=device)
    binding.nbos_policy_clip(grads, max_norm, norm, grads, norm_kind=kinds[norm_type])
    for g, dense in zip(found, grads):
        if g is not dense:
            g.copy_(dense)
    return norm
