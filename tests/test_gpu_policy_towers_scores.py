"""The towers' gradient at the rows' own hosts and beside rows that count nothing.

A row's hosts take part in the softmax with the same scores as all others: at temperatures where two summations of one product lie
many temperatures apart, a row whose best host is listed still has p = 1 there.
"""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

INF = math.inf
HALF = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


@pytest.fixture(scope="module")
def nb():
    import torch
    from paper_2503_20591_b200 import binding, build as lib_build
    lib_build.build()
    assert torch.cuda.is_available()
    binding.load_library()
    return binding


def cold(groups, rows, hosts, width, k, T, dtype, mask, seed, twins=False):
    """Rows that list their best host with a teacher weight of exp(-2) beside equal others. Host vector 0 and request 0 hold the
    constants 1 and 0: column 0 of the requests' gradient is the sum of G over a row."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t16 = getattr(torch, dtype)
    a = torch.randn((groups, rows, width), generator=gen, device="cuda").to(t16)
    b = (torch.randn((groups, hosts, width), generator=gen, device="cuda") * 2.5 / math.sqrt(width)).to(t16)
    a[..., 0], b[..., 0] = 0, 1
    if twins:
        b[:, hosts // 2:2 * (hosts // 2)] = b[:, :hosts // 2]   # every host has a twin: the best ones share p
    asks = room = None
    x = a.double() @ b.double().transpose(1, 2)
    if mask:
        asks = torch.randint(0, 9, (groups, rows, 4), generator=gen, device="cuda", dtype=torch.int32)
        room = torch.randint(3, 20, (groups, hosts, 4), generator=gen, device="cuda", dtype=torch.int32)
        if twins:
            room[:, hosts // 2:2 * (hosts // 2)] = room[:, :hosts // 2]
        x[(asks[:, :, None] > room[:, None]).any(-1)] = -INF
    ids = torch.randint(0, hosts, (groups, rows, k), generator=gen, device="cuda", dtype=torch.int32)
    ids[..., k // 2] = x.argmax(-1).int()
    teacher = torch.zeros((groups, rows, k), device="cuda")
    teacher[..., k // 2] = -2 * T
    return dict(requests=a, host_vectors=b, hosts=ids, teacher_logits=teacher, asks=asks, room=room), x


def cold_reference(c, x, T, gap):
    """(loss / T, G / T, which rows are clear) of the formula in 64 bits; rows in which another score lies within `gap` of the best are
    not clear."""
    import torch
    ids = c["hosts"].long()
    top = x.amax(-1, keepdim=True)
    alive = top > -INF
    top = torch.where(alive, top, 0.0)
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    p = torch.where(alive, ((x - top) / T).exp(), zero)
    total = p.sum(-1, keepdim=True).clamp(min=1)
    at = x.gather(2, ids)
    w = torch.where(at > -INF, (c["teacher_logits"].double() / T).exp(), zero)
    some = w.sum(-1, keepdim=True) > 0
    q = w / torch.where(some, w.sum(-1, keepdim=True), 1.0)
    G = torch.where(some, p / total, zero)
    G.scatter_add_(2, ids, -q)
    loss = torch.where(q > 0, q * (T * q.log() - (at - top) + T * total.log()), zero).sum(-1)
    second = torch.where((x == top) | (x == -INF), -INF, x).amax(-1)
    return loss, G, ~alive[..., 0] | (second < top[..., 0] - gap)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("T", [1e-36, 1e-7, 1e-6, 1e-5])
@pytest.mark.parametrize("rows,hosts,width,k,mask,twins", [(200, 700, 32, 3, False, False), (200, 700, 1024, 3, True, False), (40, 2000, 1024, 1, False, False),
                                                           (300, 515, 512, 9, False, True), (70, 300, 1024, 33, True, True), (40, 5000, 333, 33, False, False)])
def test_a_listed_host_that_is_the_best(nb, rows, hosts, width, k, mask, twins, T, dtype):
    """Scores are off by at most width 2^-23 sum |a_i b_i| =: off, so rows that are clear by 2 off + 100 T have p = 1 (or 1/2 with a
    twin, whose products are the same) at the best host and 0 elsewhere; loss / T is off by 2 off and T times 1e-5 of its parts."""
    import torch
    c, x = cold(2, rows, hosts, width, k, T, dtype, mask, rows + width, twins)
    off = width * 2.0 ** -23 * float((c["requests"].double().abs() @ c["host_vectors"].double().abs().transpose(1, 2)).max())
    loss_T, G, clear = cold_reference(c, x, T, 2 * off + 100 * T)
    assert float(clear.float().mean()) > 0.5
    loss, stats = torch.empty((2, rows), device="cuda"), torch.empty((2, rows, 2 + k), device="cuda")
    args, fit = (c["requests"], c["host_vectors"], c["hosts"], c["teacher_logits"]), dict(asks=c["asks"], room=c["room"])
    grads = [torch.empty_like(t) for t in args[:2]]
    nb.nbos_policy_towers(*args, loss, stats, temperature=T, **fit)
    nb.nbos_policy_towers_backward(*args, stats, *grads, None, 1.0 / T, T, **fit)
    if T > 1e-30:   # (the loss itself is in 32 bits)
        assert ((loss.double() / T - loss_T).abs() <= 2 * off + 1e-5 * (loss_T.abs() + 20 * T))[clear].all()
    b, half = c["host_vectors"].double(), HALF[dtype]
    want = G @ b
    # G of p and q within 1e-5, held in 16 bits (at least half a step); sums in 32 bits, their result rounded once more
    tol = (2 * half + 1e-4) * ((G.abs() + (G != 0)) @ b.abs()) + half * want.abs() + 2.0 ** -24
    assert ((grads[0].double() - want).abs() <= tol)[clear].all()
    sums = grads[0][..., 0].double().abs()   # all p of a row add up to 1, as its q do, whichever of its hosts are close
    assert (sums <= half * 4 * (1 + k)).all(), float(sums.max())
    assert torch.isfinite(grads[1]).all()


@pytest.mark.parametrize("hosts,k,mask", [(700_001, 7, False), (1 << 20, 40, True), (1 << 20, 3, False), (8192, 256, False), (8193, 256, True), (130, 256, True)])
def test_scores_at_the_entries_are_the_tables(nb, hosts, k, mask):
    """What is saved of a row's entries, up to the largest number of hosts and with lists denser than the table: whole-numbered vectors,
    so scores are exact; -inf where there is no host or no room."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(9)
    ints = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=gen, device="cuda")
    rows = 37
    a, b = ints(-3, 4, 1, rows, 24).bfloat16(), ints(-3, 4, 1, hosts, 24).bfloat16()
    ids = ints(-2, hosts + 2, 1, rows, k).int()
    ids[0, :, 0] = hosts - 1
    ids[0, 5] = ids[0, 5, 0]              # one host over and over
    asks, room = (ints(0, 9, 1, rows, 4).int(), ints(3, 20, 1, hosts, 4).int()) if mask else (None, None)
    if mask:
        asks[0, 7, 2] = -1
    stats = torch.full((1, rows, 2 + k), -7.0, device="cuda")
    nb.nbos_policy_towers(a, b, ids, None, None, stats, asks=asks, room=room)
    there = (ids >= 0) & (ids < hosts)
    at = (ids * there).long()
    if mask:
        there &= (asks[0, :, None] <= room[0, at[0]]).all(-1) & (asks[0] >= 0).all(-1)[:, None]
    want = torch.einsum("rd,rkd->rk", a[0].double(), b[0, at[0]].double())
    assert torch.equal(stats[0, :, 2:].double(), torch.where(there[0], want, -INF))
