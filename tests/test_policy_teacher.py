"""A teacher that wants a gradient is refused in Python, before any pointer is taken: it would get none, without a word."""
from __future__ import annotations

import pytest
import torch

from paper_2503_20591_b200 import policy


@pytest.mark.parametrize("shape", [(4, 3), (3,)])
def test_a_teacher_that_requires_a_gradient_is_refused(shape):
    x, hosts = torch.zeros(4, 8), torch.zeros(4, 3, dtype=torch.int32)
    teacher = torch.zeros(shape, requires_grad=True)
    with pytest.raises(ValueError, match="detach"):
        policy.distill_loss(x, hosts, teacher)
    # without a gradient in play, and detached, it is a teacher like any other: what is refused then is the CPU
    with torch.no_grad(), pytest.raises(ValueError, match="cuda"):
        policy.distill_loss(x, hosts, teacher)
    with pytest.raises(ValueError, match="cuda"):
        policy.distill_loss(x, hosts, teacher.detach())
