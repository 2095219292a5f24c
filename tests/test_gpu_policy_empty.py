"""Batches without rows, and without groups, through autograd: losses and gradients of no elements, no error."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(0, 5, 8), (3, 0, 8), (0, 8)])
def test_empty_batches_under_autograd(shape):
    import torch
    from paper_2503_20591_b200 import build as lib_build, policy
    lib_build.build()
    x = torch.zeros(shape, device="cuda", requires_grad=True)
    hosts = torch.zeros((*shape[:-1], 3), dtype=torch.int32, device="cuda")
    loss = policy.distill_loss(x, hosts)
    even, counts, shares = policy.balance_loss(x, hosts)
    drawn, found = policy.sample_hosts(x.detach(), torch.zeros((*shape[:-1], 3), device="cuda"), temperature=1.0, top_k=3)
    assert loss.shape == shape[:-1] == found.shape and drawn.shape == (*shape[:-1], 3)
    assert even.shape == shape[:-2] and counts.shape == shares.shape == (*shape[:-2], 8)
    assert not even.any() and not counts.any() and not shares.any()
    (loss.sum() + even.sum()).backward()
    assert x.grad.shape == shape
