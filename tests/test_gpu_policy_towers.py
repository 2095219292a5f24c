"""Distillation of a two-tower policy against its formula in 64 bits.

Tolerances, derived once. Vectors are 16-bit values, so products of two are exact in 32 bits.
  A logit is a sum of D products in 32 bits, each addition off by at most 2^-23 of a partial sum (the tensor cores cut off
  where others round): |dx| <= D 2^-23 sum |a_i b_i| =: dx.
  A power p = 2^((x - m) c) / S then has relative error 2 dx / T (its own x and those in S) + (160 + 6 |x|max / T) 2^-24: three
  roundings of the exponent, whose size is at most 2 |x|max log2(e) / T; the power, the sum of at most 128 additions a
  thread, 8 of the parts, and the quotient. Call it rho. q has less.
  loss: T^2 times the error of ln p and ln q, and of sums of terms of size L: T^2 (2 rho + 64 2^-24 (1 + L)).
  G = f (p - q), f = T scale grad_loss: |dG| <= f (p + q) rho + half a step of the type (2^-8 |G| in bf16, 2^-11 |G| in f16; below
  f16's normal numbers half of its smallest step, 2^-25, over the factor that G carries, at least 2^14 / max f).
  Up to 64 rows a group G is held as two values, the second what the first's rounding took: half a step of half a step.
  da = G b: |dG| |b| + (H + 64) 2^-23 |G| |b| (sums in 32 bits) + half a step of the result. db alike.
"""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

HALF = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
INF = math.inf


@pytest.fixture(scope="module")
def nb():
    import torch
    from paper_2503_20591_b200 import binding, build as lib_build
    lib_build.build()
    assert torch.cuda.is_available()
    binding.load_library()
    return binding


def make(groups, rows, hosts, width, k, dtype, mask, seed, pad=0, shift=0):
    """Inputs on the GPU; rows `pad` values apart beyond their width, the first `shift` values after an allocation's start."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    ints = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=gen, device="cuda", dtype=torch.int32)

    def vectors(n, scale):
        buf = torch.full((groups * n * (width + pad) + shift,), 7.0, dtype=getattr(torch, dtype), device="cuda")
        t = buf[shift:].view(groups, n, width + pad)[..., :width]
        t.copy_(rand(groups, n, width) * scale)
        return t

    c = dict(requests=vectors(rows, 1.0), host_vectors=vectors(hosts, 2.5 / math.sqrt(width)))
    ids = ints(-1, hosts, groups, rows, k)
    if rows > 2:
        ids[:, 0] = -1                     # a row without entries
        ids[:, 1, -1] = hosts              # beyond the table
        if k > 1:
            ids[:, 2, 1] = ids[:, 2, 0]    # listed twice
    c["hosts"] = ids
    c["teacher_logits"] = 2 * rand(groups, rows, k)
    if k > 2:
        c["teacher_logits"][..., 2] = -INF
    c["asks"] = c["room"] = None
    if mask:
        c["asks"], c["room"] = ints(0, 9, groups, rows, 4), ints(3, 20, groups, hosts, 4)
        if rows > 4:
            c["asks"][:, 3, 1] = 20        # fits nowhere
            c["asks"][:, 4, 2] = -1        # nor does that
    return c


def reference(c, T, f, values=1):
    """loss, G's two products, and their tolerances, in 64 bits, one group at a time (f: factor of each row's gradient; G is held as
    so many `values`)."""
    import torch
    out = []
    half = HALF[str(c["requests"].dtype)[6:]]
    small = half == HALF["float16"]
    for g in range(c["requests"].shape[0]):
        a, b = c["requests"][g].double(), c["host_vectors"][g].double()
        n, width = b.shape
        x, size = a @ b.T, a.abs() @ b.abs().T
        if c["asks"] is not None:
            asks, room = c["asks"][g], c["room"][g]
            x[(asks[:, None] > room[None]).any(-1) | (asks < 0).any(-1)[:, None]] = -INF
        ids = c["hosts"][g].long()
        inside = (ids >= 0) & (ids < n)
        ids = ids * inside
        at = x.gather(1, ids)
        t = torch.zeros_like(at) if c["teacher_logits"] is None else c["teacher_logits"][g].double()
        there = inside & (at > -INF) & (t > -INF)
        some = there.any(1, keepdim=True)
        zero = torch.zeros((), dtype=torch.float64, device=x.device)
        top = x.amax(1, keepdim=True)
        lse = torch.where(top > -INF, torch.logsumexp(x / T, 1, keepdim=True), zero)
        p = torch.where(some, (x / T - lse).exp(), zero)
        tt = torch.where(there, t / T, -INF)
        log_q = tt - torch.where(some, torch.logsumexp(tt, 1, keepdim=True), zero)
        q = torch.where(there, log_q.exp(), zero)
        log_p = at / T - lse
        loss = T * T * torch.where(there & (q > 0), q * (log_q - log_p), zero).sum(1)

        finite = torch.where(x > -INF, x, zero)
        xmax = finite.abs().amax(1, keepdim=True)
        rho = 2 * width * 2.0 ** -23 * size.amax(1, keepdim=True) / T + (160 + 6 * xmax / T) * 2.0 ** -24
        spread = torch.where(there, (log_q - log_p).abs() + log_p.abs(), zero).amax(1)
        tol_loss = T * T * (2 * rho[:, 0] + 64 * 2.0 ** -24 * (1 + spread))
        G = p.clone()
        G.scatter_add_(1, ids, -q)
        Q = torch.zeros_like(G).scatter_add_(1, ids, q)
        G *= f[g][:, None]
        dG = f[g].abs()[:, None] * (p + Q) * rho + half ** values * G.abs()
        if small:
            dG += 2.0 ** -25 * 2.0 ** -14 * f.abs().max()
        last = 2.0 ** -25 if small else 2.0 ** -133
        da, db = G @ b, G.T @ a
        tol_a = dG @ b.abs() + (n + 64) * 2.0 ** -23 * (G.abs() @ b.abs()) + half * da.abs() + last
        tol_b = dG.T @ a.abs() + (len(a) + 64) * 2.0 ** -23 * (G.abs().T @ a.abs()) + half * db.abs() + last
        out.append((loss, tol_loss, da, tol_a, db, tol_b))
    return [torch.stack(v) for v in zip(*out)]


def close(got, want, tol):
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4], want[bad][:4], tol[bad][:4])


def run(nb, c, T, scale, grad_loss, want=("a", "b")):
    import torch
    shape = c["hosts"].shape[:-1]
    fit = dict(asks=c["asks"], room=c["room"])
    loss = torch.full(shape, -7.0, device="cuda")
    stats = torch.full((*shape, 2 + c["hosts"].shape[-1]), -7.0, device="cuda")
    args = (c["requests"], c["host_vectors"], c["hosts"], c["teacher_logits"])
    nb.nbos_policy_towers(*args, loss, stats, temperature=T, **fit)
    da = torch.full(c["requests"].shape, -7.0, dtype=c["requests"].dtype, device="cuda") if "a" in want else None
    db = torch.full(c["host_vectors"].shape, -7.0, dtype=c["requests"].dtype, device="cuda") if "b" in want else None
    nb.nbos_policy_towers_backward(*args, stats, da, db, grad_loss, scale, T, **fit)
    assert nb.nbos_policy_towers_status() == nb.NBOS_OK
    return loss, da, db


def check(nb, c, T=1.0, scale=1.0, grad_loss=None, values=1):
    import torch
    shape = c["hosts"].shape[:-1]
    f = torch.full(shape, T * scale, dtype=torch.float64, device="cuda")
    if grad_loss is not None:
        f = f * grad_loss.double()
    loss, da, db = run(nb, c, T, scale, grad_loss)
    want = reference(c, T, f, values)
    close(loss, *want[:2])
    close(da, *want[2:4])
    close(db, *want[4:])
    return loss, da, db


# one of everything, tile and stage borders, odd widths, few rows and many hosts, many rows and few hosts
SIZES = [(1, 1, 1, 1), (1, 2, 3, 8), (2, 5, 1, 7), (1, 7, 33, 64), (3, 33, 77, 13), (1, 255, 257, 65), (1, 257, 255, 128),
         (2, 300, 512, 129), (1, 129, 1000, 200), (1, 1, 20000, 64), (1, 5000, 3, 32), (1, 700, 700, 513), (5, 64, 64, 1000),
         (1, 64, 4096, 2049)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("groups,rows,hosts,width", SIZES)
def test_matches_the_formula(nb, groups, rows, hosts, width, mask, dtype):
    import torch
    for i, (k, T, pad, shift) in enumerate(((3, 1.0, 0, 0), (1, 0.7, 3, 1), (33, 2.0, 8, 0))):
        c = make(groups, rows, hosts, width, k, dtype, mask, 100 * i + rows + width, pad, shift)
        gl = torch.rand((groups, rows), device="cuda") + 0.5 if i != 1 else None
        check(nb, c, T, 8.0 if dtype == "float16" else 1.0 / rows, gl)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("mask,k", [(False, 1), (True, 4), (False, 9)])
@pytest.mark.parametrize("groups,rows,hosts,width", [(1, 1, 300, 16), (1, 3, 5000, 24), (3, 2, 64, 8), (7, 33, 700, 65), (2, 64, 257, 16), (1, 64, 40000, 32)])
def test_gradients_of_few_rows(nb, groups, rows, hosts, width, mask, k, dtype):
    """What the first rounding of G takes off is not lost, the entries' included."""
    c = make(groups, rows, hosts, width, k, dtype, mask, rows + width)
    check(nb, c, 1.0, 8.0 if dtype == "float16" else 1.0, None, values=2)


@pytest.mark.parametrize("groups,rows,hosts,width,what", [(1, 4099, 70001, 72, "runs of hosts"), (1, 70003, 4099, 72, "runs of rows"),
                                                           (5, 1500, 40001, 64, "four groups, then one")])
def test_gradients_in_pieces(nb, groups, rows, hosts, width, what):
    """Scores beyond 512 MB: their gradient exists in pieces (with a shorter one at the end), whose products add up."""
    check(nb, make(groups, rows, hosts, width, 3, "bfloat16", True, 5), 1.0, 1.0)


@pytest.mark.parametrize("T", [1e-36, 1e-3, 50.0])
@pytest.mark.parametrize("mask,k", [(False, 3), (True, 3), (False, 9)])
def test_temperatures(nb, T, mask, k):
    """Far below 1 all weight is on the best host: p is 0 or 1 wherever two logits differ by more than 200 T. Rows whose two best, or
    whose entries' best teacher logits, are that close are left out of the comparison (logits are compared exactly there)."""
    import torch
    c = make(1, 200, 700, 32, k, "bfloat16", mask, 21)
    scale = 1.0 / T if T < 1 else 1.0
    if T > 1e-30:
        check(nb, c, T, scale)
        return
    loss, da, db = run(nb, c, T, scale, None)
    a, b = c["requests"][0].double(), c["host_vectors"][0].double()
    x = a @ b.T
    if mask:
        x[(c["asks"][0][:, None] > c["room"][0][None]).any(-1) | (c["asks"][0] < 0).any(-1)[:, None]] = -INF
    ids = c["hosts"][0].long()
    inside = (ids >= 0) & (ids < 700)
    at = x.gather(1, ids * inside)
    t = torch.where(inside & (at > -INF), c["teacher_logits"][0].double(), -INF)
    some = (t > -INF).any(1)
    best, teacher_best = x.argmax(1), (ids * inside).gather(1, t.argmax(1, keepdim=True))[:, 0]
    G = torch.zeros_like(x)
    rows = torch.arange(200, device="cuda")
    G[rows, best] += 1.0
    G[rows, teacher_best] -= 1.0
    G *= some[:, None]
    clear = ~some | ((x.topk(2, 1).values.diff(dim=1)[:, 0] < -1e-3) & (t.topk(2, 1).values.diff(dim=1)[:, 0] < -1e-3))
    assert int(clear.sum()) > 150
    # q = 1 at one host, ln p = (x there - the largest) / T: T^2 times that is T times the difference. A logit is off by at most
    # 32 2^-23 sum |a_i b_i| < 3e-4 (the sums stay below 70).
    want_loss = torch.where(some, x.amax(1) - x[rows, teacher_best], torch.zeros((), dtype=torch.float64, device="cuda"))
    assert ((loss[0].double() / T - want_loss).abs() <= 6e-4 + 1e-5 * want_loss)[clear].all()
    want = G @ b
    assert ((da[0].double() - want).abs() <= 3 * 2.0 ** -8 * (G.abs() @ b.abs()) + 1e-9)[clear].all()


def test_long_lists_of_hosts(nb):
    c = make(1, 60, 500, 96, 256, "float16", True, 3)
    c["hosts"][:, 5] = 17                 # one host 256 times
    check(nb, c, 1.5, 4.0)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_far_apart_rows_of_gradient(nb, dtype):
    """grad_loss over ten powers of two, zeros and signs; one row far above the others."""
    import torch
    c = make(2, 200, 300, 64, 3, dtype, False, 8)
    gl = 2.0 ** -torch.randint(0, 10, (2, 200), device="cuda").float()
    gl[:, ::5] = 0
    gl[:, 1::3] *= -1
    check(nb, c, 1.0, 1.0, gl)


def test_no_teacher_logits_and_one_list_for_all(nb):
    import torch
    c = make(2, 90, 130, 40, 3, "bfloat16", True, 4)
    c["teacher_logits"] = None
    check(nb, c)
    one = torch.tensor([2.0, 1.0, 0.0], device="cuda")
    c["teacher_logits"] = one
    a = run(nb, c, 1.0, 1.0, None)
    c["teacher_logits"] = one.expand(2, 90, 3).contiguous()
    for got, want in zip(a, run(nb, c, 1.0, 1.0, None)):
        assert torch.equal(got, want)


def test_one_gradient_is_the_same_as_both(nb):
    import torch
    c = make(2, 300, 400, 100, 3, "bfloat16", True, 9)
    both = run(nb, c, 1.0, 1.0, None)
    assert torch.equal(run(nb, c, 1.0, 1.0, None, "a")[1], both[1])
    assert torch.equal(run(nb, c, 1.0, 1.0, None, "b")[2], both[2])


def test_same_bits_every_time(nb):
    import torch
    c = make(1, 1000, 5000, 200, 3, "bfloat16", True, 10)
    c["hosts"][...] = c["hosts"] % 7      # crowded hosts
    first = run(nb, c, 1.0, 1.0, None)
    for _ in range(3):
        for got, want in zip(run(nb, c, 1.0, 1.0, None), first):
            assert torch.equal(got, want)


def test_agrees_with_distillation_on_the_table(nb):
    """The table of logits through nbos_policy_distill, where it can be stored."""
    import torch
    from paper_2503_20591_b200 import policy
    c = make(2, 120, 260, 48, 3, "bfloat16", True, 11)
    fits = (c["asks"][:, :, None] <= c["room"][:, None]).all(-1) & (c["asks"] >= 0).all(-1)[..., None]
    x = (c["requests"].double() @ c["host_vectors"].double().transpose(1, 2)).masked_fill(~fits, -INF).float()
    want = policy.distill_loss(x, c["hosts"], c["teacher_logits"])
    got = policy.tower_distill_loss(**c)
    # both sides are within the derived bound of the formula
    tol = reference(c, 1.0, torch.ones(2, 120, dtype=torch.float64, device="cuda"))[1]
    close(got, want.double(), 2 * tol)


def test_rows_that_count_nothing(nb):
    """No entries, or none that fits: loss and gradient 0, whatever the row's vector holds."""
    import torch
    c = make(1, 40, 50, 24, 2, "bfloat16", True, 12)
    c["hosts"][0, :10] = -1
    c["asks"][0, 10:20] = 100
    c["teacher_logits"][0, 20:30] = -INF
    c["teacher_logits"][0, 25:30, 0] = math.nan
    loss, da, db = check(nb, c)
    assert (loss[0, :30] == 0).all() and (da[0, :30] == 0).all()
    c["requests"][0, 5] = math.nan
    loss, da, _ = run(nb, c, 1.0, 1.0, None, "a")
    assert (loss[0, :30] == 0).all() and (da[0, :30] == 0).all()


def test_masked_hosts_may_hold_anything(nb):
    """NaN and infinities in the vector of a host that nothing fits change neither loss nor the requests' statistics."""
    import torch
    c = make(1, 70, 300, 32, 3, "float16", True, 13)
    c["room"][0, 100:110] = -1
    before = run(nb, c, 1.0, 1.0, None)
    c["host_vectors"][0, 100:105] = math.nan
    c["host_vectors"][0, 105:110] = INF
    loss, _, db = run(nb, c, 1.0, 1.0, None, "b")
    assert torch.equal(loss, before[0]) and torch.equal(db, before[2])


def test_a_row_that_is_not_finite_spoils_itself(nb):
    import torch
    c = make(1, 30, 300, 32, 3, "bfloat16", False, 14)
    c["hosts"][...] = torch.arange(3, device="cuda", dtype=torch.int32)
    before = run(nb, c, 1.0, 1.0, None, "a")
    c["requests"][0, 11, 5] = math.nan
    loss, da, _ = run(nb, c, 1.0, 1.0, None, "a")
    rest = torch.arange(30, device="cuda") != 11
    assert loss[0, 11].isnan() and da[0, 11].isnan().all()
    assert torch.equal(loss[0, rest], before[0][0, rest]) and torch.equal(da[0, rest], before[1][0, rest])


@pytest.mark.parametrize("k", [3, 9])
def test_a_teacher_logit_that_is_infinite_spoils_its_row(nb, k):
    """Its weight is inf / inf, whichever kernel puts the row's entries in."""
    import torch
    c = make(1, 30, 300, 32, k, "float16", False, 22)
    c["hosts"][...] = torch.arange(k, device="cuda", dtype=torch.int32)
    before = run(nb, c, 1.0, 1.0, None, "a")
    c["teacher_logits"][0, 11, 0] = INF
    loss, da, _ = run(nb, c, 1.0, 1.0, None, "a")
    rest = torch.arange(30, device="cuda") != 11
    assert loss[0, 11].isnan() and da[0, 11].isnan().all()
    assert torch.equal(loss[0, rest], before[0][0, rest]) and torch.equal(da[0, rest], before[1][0, rest])


def test_one_table_of_hosts_for_all_groups(nb):
    """A group stride of 0 is read as it is; autograd adds the groups' gradients up."""
    import torch
    from paper_2503_20591_b200 import policy
    c = make(3, 100, 150, 40, 3, "bfloat16", True, 15)
    c["host_vectors"] = c["host_vectors"][:1].expand(3, -1, -1)
    check(nb, c)
    leaf = c["host_vectors"][0].clone().requires_grad_(True)
    policy.tower_distill_loss(**dict(c, host_vectors=leaf.expand(3, -1, -1))).sum().backward()
    _, _, db = run(nb, c, 1.0, 1.0, None, "b")
    torch.testing.assert_close(leaf.grad, db.sum(0), rtol=2.0 ** -6, atol=0.05)   # three roundings to bf16 of values below 4


def test_autograd_and_differences(nb):
    """The gradient of a weighted sum of losses against differences of the loss in 64 bits along random directions."""
    import torch
    from paper_2503_20591_b200 import policy
    c = make(2, 50, 80, 32, 3, "float16", True, 16)
    w = torch.rand(2, 50, device="cuda") + 0.5
    a, b = (c[n].clone().requires_grad_(True) for n in ("requests", "host_vectors"))
    loss = policy.tower_distill_loss(**dict(c, requests=a, host_vectors=b), temperature=1.3)
    (loss * w).sum().backward()

    def value(x, y):
        f = torch.zeros(2, 50, dtype=torch.float64, device="cuda")
        return float((reference(dict(c, requests=x, host_vectors=y), 1.3, f)[0] * w).sum())

    class In64:   # 64-bit vectors under a 16-bit name, for the reference
        def __init__(self, t):
            self.t, self.dtype, self.shape = t, torch.float16, t.shape

        def __getitem__(self, g):
            return self.t[g]

    for leaf, first in ((a, True), (b, False)):
        d = torch.randn(leaf.shape, device="cuda").double()
        e = 1e-4
        pair = lambda s: (In64(a.detach().double() + s * d), In64(b.detach().double())) if first else \
            (In64(a.detach().double()), In64(b.detach().double() + s * d))
        slope = (value(*pair(e)) - value(*pair(-e))) / (2 * e)
        got = float((leaf.grad.double() * d).sum())
        # G and the gradient are each off by at most 2^-11 relative; differences by their third order, below 1e-6
        size = float((leaf.grad.double().abs() * d.abs()).sum())
        assert abs(got - slope) <= 2.0 ** -9 * size + 1e-5


def test_empty_batches(nb):
    import torch
    e = lambda *s, t=torch.bfloat16: torch.full(s, -7.0, device="cuda").to(t)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    # no rows: the hosts' gradient is 0
    db = e(2, 30, 8)
    nb.nbos_policy_towers(e(2, 0, 8), e(2, 30, 8), i32(2, 0, 3), None, e(2, 0, t=torch.float32))
    nb.nbos_policy_towers_backward(e(2, 0, 8), e(2, 30, 8), i32(2, 0, 3), None, e(2, 0, 5, t=torch.float32), e(2, 0, 8), db)
    assert (db == 0).all()
    # no groups: nothing at all
    nb.nbos_policy_towers(e(0, 4, 8), e(0, 30, 8), i32(0, 4, 3), None, e(0, 4, t=torch.float32))
    nb.nbos_policy_towers_backward(e(0, 4, 8), e(0, 30, 8), i32(0, 4, 3), None, e(0, 4, 5, t=torch.float32), e(0, 4, 8), e(0, 30, 8))


def test_gradients_with_gaps_leave_them_alone(nb):
    import torch
    c = make(2, 60, 70, 24, 3, "bfloat16", False, 17)
    want = run(nb, c, 1.0, 1.0, None)
    loss, stats = torch.empty(2, 60, device="cuda"), torch.empty(2, 60, 5, device="cuda")
    args = (c["requests"], c["host_vectors"], c["hosts"], c["teacher_logits"])
    nb.nbos_policy_towers(*args, loss, stats)
    ga, gb = torch.full((2, 64, 31), -7.0, device="cuda").bfloat16(), torch.full((2, 75, 29), -7.0, device="cuda").bfloat16()
    nb.nbos_policy_towers_backward(*args, stats, ga[:, :60, 3:27], gb[:, 2:72, :24])
    assert torch.equal(ga[:, :60, 3:27], want[1]) and torch.equal(gb[:, 2:72, :24], want[2])
    ga[:, :60, 3:27], gb[:, 2:72, :24] = -7.0, -7.0
    assert (ga == -7.0).all() and (gb == -7.0).all()


def test_streams_and_graphs(nb):
    """On a stream of its own, and captured with two inputs and replayed with others; an eager graph of the same leaves lives."""
    import torch
    from paper_2503_20591_b200 import policy
    c, d = (make(2, 300, 400, 64, 3, "bfloat16", True, s) for s in (18, 19))
    want = [run(nb, x, 1.0, 1.0, None) for x in (c, d)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run(nb, c, 1.0, 1.0, None)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(got, want[0]))

    a, b = c["requests"].clone().requires_grad_(True), c["host_vectors"].clone().requires_grad_(True)
    alive = policy.tower_distill_loss(**dict(c, requests=a, host_vectors=b)).sum()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        stats, loss = torch.empty(2, 300, 5, device="cuda"), torch.empty(2, 300, device="cuda")
        ga, gb = torch.empty_like(a), torch.empty_like(b)
        with torch.cuda.graph(graph):
            args = (a.detach(), b.detach(), c["hosts"], c["teacher_logits"])
            nb.nbos_policy_towers(*args, loss, stats, asks=c["asks"], room=c["room"])
            nb.nbos_policy_towers_backward(*args, stats, ga, gb, asks=c["asks"], room=c["room"])
        graphs.append((graph, loss, ga, gb))
    with torch.no_grad():
        a.copy_(d["requests"]), b.copy_(d["host_vectors"])
        for n in ("hosts", "teacher_logits", "asks", "room"):
            c[n].copy_(d[n])
    for graph, *_ in graphs:
        graph.replay()
    torch.cuda.synchronize()
    for _, *got in graphs:
        assert all(torch.equal(x, y) for x, y in zip(got, want[1]))
    del alive


@pytest.mark.parametrize("rows,k", [(30, 3), (300, 9)])
def test_captured_with_a_gradient_for_each_row(nb, rows, k):
    """Forward and backward in one graph, whose factor follows the grad_loss of each replay."""
    import torch
    c = make(2, rows, 400, 44, k, "float16", True, 23)
    gl = torch.rand(2, rows, device="cuda") + 0.5
    stats, loss = torch.empty(2, rows, 2 + k, device="cuda"), torch.empty(2, rows, device="cuda")
    grads = [torch.empty_like(c[n], memory_format=torch.contiguous_format) for n in ("requests", "host_vectors")]
    args, fit = (c["requests"], c["host_vectors"], c["hosts"], c["teacher_logits"]), dict(asks=c["asks"], room=c["room"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nb.nbos_policy_towers(*args, loss, stats, **fit)
        nb.nbos_policy_towers_backward(*args, stats, *grads, gl, **fit)
    for factor in (1.0, 1000.0, 2.0 ** -9):
        gl *= factor
        want = run(nb, c, 1.0, 1.0, gl)
        for t in (loss, *grads):
            t.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((loss, *grads), want))
