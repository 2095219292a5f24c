"""How many 16-bit values hold an entry of the scores' gradient G, and what that does to the towers' gradients.

Bounds: those of test_gpu_policy_towers for one value and for two. Where a row's terms cancel those say little, so there the 2-norm of
the error is compared with that of the exact gradient rounded once. Vectors are whole numbers then, and scores exact: what is left is
the second value's rounding (2^-8 of the first's) and the power's and sum's of p (some 2^-22), times the common part's eleven: below a
tenth of a rounding in either type, and errors that do not go together add in squares.
"""
from __future__ import annotations

import math

import pytest

from test_gpu_policy_towers import close, make, nb, reference   # noqa: F401 (nb is a fixture)

pytestmark = pytest.mark.gpu


def both(nb, c, T, scale, values):
    import torch
    shape, k = c["hosts"].shape[:-1], c["hosts"].shape[-1]
    loss, stats = torch.empty(shape, device="cuda"), torch.empty((*shape, 2 + k), device="cuda")
    args, fit = (c["requests"], c["host_vectors"], c["hosts"], c["teacher_logits"]), dict(asks=c["asks"], room=c["room"])
    grads = [torch.empty_like(t, memory_format=torch.contiguous_format) for t in args[:2]]
    nb.nbos_policy_towers(*args, loss, stats, temperature=T, **fit)
    nb.nbos_policy_towers_backward(*args, stats, *grads, None, scale, T, **fit, **({} if values is None else dict(gradient_values=values)))
    return grads


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("values", [1, 2, None])
@pytest.mark.parametrize("groups,rows,hosts,width,k,mask", [(1, 1, 300, 16, 3, False), (3, 33, 77, 13, 1, True), (2, 65, 257, 24, 4, True), (1, 600, 900, 40, 3, False),
                                                            (1, 3000, 5, 32, 2, False), (2, 300, 1000, 130, 9, True)])
def test_within_the_bound_of_each(nb, groups, rows, hosts, width, k, mask, values, dtype):
    import torch
    c = make(groups, rows, hosts, width, k, dtype, mask, rows + width)
    scale = 8.0 if dtype == "float16" else 1.0
    want = reference(c, 1.0, torch.full((groups, rows), scale, dtype=torch.float64, device="cuda"), values or 2)
    for got, ref, tol in zip(both(nb, c, 1.0, scale, values), want[2::2], want[3::2]):
        close(got, ref, tol)


@pytest.mark.parametrize("dtype,scale", [("bfloat16", 1.0), ("float16", 4.0)])
@pytest.mark.parametrize("rows,hosts,k,mask", [(200, 700, 3, False), (1000, 4000, 9, True), (20, 600, 1, False), (700, 40, 3, True)])
def test_what_vectors_have_in_common_cancels(nb, rows, hosts, k, mask, dtype, scale):
    """Host vectors whose common part is eleven times what tells them apart: a row's p - q add up to 0, and so does what it brings."""
    import torch
    c = make(1, rows, hosts, 32, k, dtype, mask, 3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    ints = lambda *s: torch.randint(-2, 3, s, generator=gen, device="cuda").to(getattr(torch, dtype))
    c["requests"], c["host_vectors"] = ints(1, rows, 32), ints(1, hosts, 32) + 16
    want = reference(c, 4.0, torch.full((1, rows), 4 * scale, dtype=torch.float64, device="cuda"))
    once = [(w.to(c["requests"].dtype).double() - w).norm() for w in want[2::2]]
    off = [(g.double() - w).norm() for g, w in zip(both(nb, c, 4.0, scale, None), want[2::2])]
    assert all(o <= 1.1 * r for o, r in zip(off, once)), (off, once)
    # with one value the requests' gradient is several times as far off
    coarse = (both(nb, c, 4.0, scale, 1)[0].double() - want[2]).norm()
    assert 3 * off[0] < coarse


def test_through_autograd(nb):
    import torch
    from paper_2503_20591_b200 import policy
    c = make(2, 100, 300, 40, 3, "bfloat16", True, 5)
    for values in (1, 2):
        leaves = [c[n].clone().requires_grad_(True) for n in ("requests", "host_vectors")]
        loss = policy.tower_distill_loss(*leaves, c["hosts"], c["teacher_logits"], 1.0, c["asks"], c["room"], gradient_values=values)
        loss.sum().backward()
        assert all(torch.equal(t.grad, g) for t, g in zip(leaves, both(nb, c, 1.0, 1.0, values)))
