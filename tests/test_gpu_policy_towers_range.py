"""Which rows the range of G follows: those that count, by what is finite."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

INF = math.inf


@pytest.fixture(scope="module")
def nb():
    import torch
    from paper_2503_20591_b200 import binding, build as lib_build
    lib_build.build()
    assert torch.cuda.is_available()
    binding.load_library()
    return binding


def make(rows, k, dtype, mask, seed):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")
    ints = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=gen, device="cuda", dtype=torch.int32)
    t16 = getattr(torch, dtype)
    return dict(requests=rand(1, rows, 64).to(t16), host_vectors=(rand(1, 300, 64) / 3).to(t16), hosts=ints(0, 300, 1, rows, k),
                teacher_logits=rand(1, rows, k), asks=ints(0, 9, 1, rows, 4) if mask else None, room=ints(3, 20, 1, 300, 4) if mask else None)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("rows,k", [(40, 3), (200, 3), (200, 9)])
def test_what_arrives_at_rows_that_count_nothing_changes_no_other(nb, rows, k, dtype):
    """A row without a counting entry has gradient 0 whatever arrives at its loss, and the others' range does not follow it."""
    import torch
    c = make(rows, k, dtype, True, 3)
    c["hosts"][0, :10] = -1
    c["asks"][0, 10:20] = 100
    c["teacher_logits"][0, 20:30] = -INF
    loss, stats = torch.empty((1, rows), device="cuda"), torch.empty((1, rows, 2 + k), device="cuda")
    args, fit = (c["requests"], c["host_vectors"], c["hosts"], c["teacher_logits"]), dict(asks=c["asks"], room=c["room"])
    nb.nbos_policy_towers(*args, loss, stats, **fit)
    grad_loss = torch.rand((1, rows), device="cuda") + 0.5

    def grads():
        out = [torch.empty_like(t) for t in args[:2]]
        nb.nbos_policy_towers_backward(*args, stats, *out, grad_loss, 1.0, 1.0, **fit)
        return out

    want = grads()
    assert (want[0][0, :30] == 0).all() and (want[0][0, 30:] != 0).any()
    for odd in (1e30, INF, -INF, math.nan, 0.0):
        grad_loss[0, :30:3] = odd
        assert all(torch.equal(x, y) for x, y in zip(grads(), want)), odd


@pytest.mark.parametrize("odd", [INF, -INF, math.nan])
def test_what_is_not_finite_spoils_its_own_row(nb, odd):
    """A row whose arriving gradient is not finite has no use for a range; the other requests' gradients keep theirs, beyond 65,504 too."""
    import torch
    c = make(200, 3, "float16", False, 4)
    loss, stats = torch.empty((1, 200), device="cuda"), torch.empty((1, 200, 5), device="cuda")
    args = (c["requests"], c["host_vectors"], c["hosts"], c["teacher_logits"])
    nb.nbos_policy_towers(*args, loss, stats)
    grad_loss = torch.rand((1, 200), device="cuda") * 2.0 ** -14 + 2.0 ** -14

    def grad():
        out = torch.empty_like(c["requests"])
        nb.nbos_policy_towers_backward(*args, stats, out, None, grad_loss, 1.0)
        return out

    want = grad()
    at = int(grad_loss.argmin())   # (not the one that the range follows)
    grad_loss[0, at] = odd
    got = grad()
    rest = torch.arange(200, device="cuda") != at
    assert torch.equal(got[0, rest], want[0, rest]) and not torch.isfinite(got[0, at]).all()
