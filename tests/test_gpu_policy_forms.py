"""Every form of the policy kernels with several rows for each of its warps, blocks and clusters, so that rows on their way, stages that
are used again and writes that are put off all happen: against the formulas in 64 bits on the GPU, within the tolerances
that test_gpu_policy.py derives. Warps of short rows: 2 or 3 blocks of 8 on each of 148 SMs; blocks of longer ones: 1 to 12 an SM."""
from __future__ import annotations

import math

import numpy as np
import pytest

from test_gpu_policy import DTYPES, E, HALF_ULP, SMALLEST, TOL_P, nb, run_sample, settings, torch_sample  # noqa: F401 (nb is a fixture)

pytestmark = pytest.mark.gpu
INF = math.inf


def logits_of(gen, rows, n, dtype, pad=0, shift=0):
    """A table whose rows are n + pad apart and begin `shift` elements into it, a tenth of the hosts out, some rows empty; and a second
    one laid out alike."""
    import torch

    def empty():
        buf = torch.full((rows * (n + pad) + shift,), 99.0, dtype=getattr(torch, dtype), device="cuda")
        return buf[shift:].view(rows, n + pad)[:, :n]

    x = empty()
    v = torch.randn((rows, n), generator=gen, device="cuda").mul_(2.5)
    v.masked_fill_(torch.rand((rows, n), generator=gen, device="cuda") < 0.1, -INF)
    v[:: 101] = -INF
    x.copy_(v)
    return x, empty


def hosts_of(gen, rows, n, k):
    """-1 and ids beyond the table among them, hosts listed twice, rows without any."""
    import torch
    h = torch.randint(0, n + 1 + n // 50, (rows, k), generator=gen, device="cuda")
    h[torch.rand((rows, k), generator=gen, device="cuda") < 0.15] = -1
    h[:: 7, k - 1] = h[:: 7, 0]
    h[3:: 13] = -1
    return h.int()


def softmax64(x):
    import torch
    lse = torch.logsumexp(x, -1, keepdim=True)
    log_p = torch.where(lse == -INF, -INF, x - lse)
    return log_p.exp(), log_p


def within(got, want, tol):
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist())


# ---- distillation ---------------------------------------------------------------------------------------------------
def distill64(x, hosts, teacher, T, mult):
    """(loss, its tolerance, gradient times mult, the p + q that its tolerance scales with)"""
    import torch
    n = x.shape[1]
    inside = (hosts >= 0) & (hosts < n)
    ids = torch.where(inside, hosts, 0).long()
    p, log_p = softmax64(x.double() / T)
    at = log_p.gather(1, ids)
    there = inside & (at > -INF) & (teacher > -INF)
    q, log_q = softmax64(torch.where(there, teacher.double() / T, -INF))
    some = there.any(1, keepdim=True)
    loss = T * T * torch.where(q > 0, q * (log_q - at), 0.0).sum(1)
    spread = torch.where(there, log_q.abs() + at.abs(), 0.0).amax(1)
    tol = 512 * E * (1 + spread) * T * T
    spread_q = torch.zeros_like(p).scatter_add_(1, ids, torch.where(there, q, 0.0))
    p = p * some
    return loss, tol, (p - spread_q) * (T * mult[:, None]), (p + spread_q) * (T * mult[:, None].abs())


WARP_ROWS = [(150000, 5), (120000, 33), (60000, 150), (120000, 250), (60000, 300), (20000, 600), (20000, 1000), (20000, 1024)]
BLOCK_ROWS = [(7200, 1025), (3600, 3000), (2400, 4099), (1300, 7000), (600, 16384)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,n", WARP_ROWS + BLOCK_ROWS)
def test_distill_with_several_rows_a_team(nb, rows, n, dtype):  # noqa: F811
    import torch
    gen = torch.Generator(device="cuda").manual_seed(rows + n)
    for k, T, pad, shift in ((3, 1.0, 0, 0), (3, 0.7, 3, 1), (70, 1.5, 8, 0)):
        x, empty = logits_of(gen, rows, n, dtype, pad, shift)
        hosts = hosts_of(gen, rows, n, k)
        teacher = torch.randn((rows, k), generator=gen, device="cuda") * 2
        teacher[torch.rand((rows, k), generator=gen, device="cuda") < 0.05] = -INF
        arrives, scale = torch.randn(rows, generator=gen, device="cuda"), 64.0
        want_l, tol_l, want_g, size = distill64(x, hosts, teacher, T, arrives.double() * scale)
        tol_g = TOL_P * size + want_g.abs() * (HALF_ULP[dtype] * 1.01) + SMALLEST[dtype]
        loss, stats = torch.full((rows,), -7.0, device="cuda"), torch.full((rows, 2), -7.0, device="cuda")
        grad = empty()
        nb.nbos_policy_distill(x, hosts, teacher, loss, None, arrives, scale, grad, temperature=T)
        within(loss, want_l, tol_l)
        within(grad, want_g, tol_g)
        alone, again = torch.full_like(loss, -7.0), torch.full((rows, n), 99.0, dtype=x.dtype, device="cuda")
        nb.nbos_policy_distill(x, hosts, teacher, alone, stats, temperature=T)
        assert torch.equal(alone, loss)
        nb.nbos_policy_distill_backward(x, hosts, teacher, stats, again, arrives, scale, temperature=T)
        within(again, want_g, tol_g)
        nb.nbos_policy_distill(x, hosts, teacher, alone, None, arrives, scale, x, temperature=T)     # over the logits
        assert torch.equal(alone, loss) and torch.equal(x, grad)


# ---- balance --------------------------------------------------------------------------------------------------------
def balance64(x, hosts, mult):
    """One group: loss, counts, shares, gradient times mult, what its tolerance scales with."""
    import torch
    n = x.shape[1]
    inside = (hosts >= 0) & (hosts < n)
    counts = torch.bincount(hosts[inside].long(), minlength=n)
    live = inside.any(1, keepdim=True)
    n_live = max(1, int(live.sum()))
    f = counts.double() / max(1, int(counts.sum()))
    p = softmax64(x.double())[0] * live
    dot = (p @ f)[:, None]
    shares = p.sum(0) / n_live
    return n * (f @ shares), counts.int(), shares, p * (f - dot) * (mult * n / n_live), p * (f + dot) * (abs(mult) * n / n_live)


BALANCE = [(3, 25001, 24), (2, 20000, 60), (3, 12000, 120), (3, 6700, 250), (2, 8000, 300), (3, 6000, 380), (3, 5000, 500), (3, 3300, 700),
           (3, 3300, 1000), (40, 70, 1000),
           (3, 800, 1025), (2, 400, 4099), (50, 20, 3000), (3, 250, 16384), (2, 200, 20000), (3, 60, 40001)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("groups,rows,n", BALANCE)
def test_balance_with_several_rows_a_team(nb, groups, rows, n, dtype):  # noqa: F811
    """Stretches of rows cross from one group into the next. A thread adds up 64 rows of a column at most at these sizes."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(groups + rows + n)
    for k, pad, shift in ((3, 0, 0), (2, 3, 1), (40, 8, 0)):
        flat, empty = logits_of(gen, groups * rows, n, dtype, pad, shift)
        x, grad = flat.unflatten(0, (groups, rows)), empty().unflatten(0, (groups, rows))
        hosts = hosts_of(gen, groups * rows, n, k).view(groups, rows, k)
        hosts[groups // 2, :, 1:] = -1
        arrives, scale = torch.randn(groups, generator=gen, device="cuda"), 512.0 * rows / n
        loss, counts = torch.full((groups,), -7.0, device="cuda"), torch.full((groups, n), -7, dtype=torch.int32, device="cuda")
        shares, stats = torch.full((groups, n), -7.0, device="cuda"), torch.full((groups, rows, 2), -7.0, device="cuda")
        nb.nbos_policy_balance(x, hosts, loss, counts, shares, stats, arrives, scale, grad)
        again = torch.full(x.shape, 99.0, dtype=x.dtype, device="cuda")
        nb.nbos_policy_balance_backward(x, hosts, stats, again, arrives, scale)
        for g in range(groups):
            want = balance64(x[g], hosts[g], float(arrives[g]) * scale)
            assert torch.equal(counts[g], want[1])
            rel = TOL_P + 64 * E
            within(shares[g], want[2], want[2] * rel + E * 2.0 ** -100)
            within(loss[g], want[0], want[0] * rel)
            tol = 2 * TOL_P * want[4] + want[3].abs() * (HALF_ULP[dtype] * 1.01) + SMALLEST[dtype]
            within(grad[g], want[3], tol)
            within(again[g], want[3], tol)
        alone = [torch.full_like(v, -7) for v in (loss, counts, shares)]
        nb.nbos_policy_balance(x, hosts, *alone)
        for v, w in zip(alone, (loss, counts, shares)):
            assert torch.equal(v, w)
        nb.nbos_policy_balance(x, hosts, *alone, None, arrives, scale, x)     # over the logits
        for v, w in zip((*alone, x), (loss, counts, shares, grad)):
            assert torch.equal(v, w)


# ---- sampling -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,n", [(1500, 1500), (1500, 2048), (1500, 4096), (1200, 4001), (40, 262145)])
def test_sample_with_many_long_rows(nb, rows, n, dtype):  # noqa: F811
    """One warp for a row of up to 4,096 hosts; rows that take turns in the workspace."""
    import torch
    rng = np.random.default_rng(rows + n)
    gen = torch.Generator(device="cuda").manual_seed(n)
    for pad, shift in ((0, 0), (3, 1)):
        x, _ = logits_of(gen, rows, n, dtype, pad, shift)
        u = rng.random((rows, 3)).astype(np.float32)
        T, k, p, q = settings(rng, rows, n, exact=False)
        for kw in (dict(), dict(top_k=k), dict(top_p=p, temperature=T), dict(temperature=T, top_k=k, top_p=p, min_p=q)):
            got, want = run_sample(nb, x, u, **kw), torch_sample(x, u, **kw)
            np.testing.assert_array_equal(got[0], want[0])
            np.testing.assert_array_equal(got[1], want[1])


# ---- as many hosts a row as there may be --------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,n", [(5000, 24), (5000, 400), (2000, 1000), (1300, 3000), (20, 20000)])
def test_256_hosts_a_row(nb, rows, n, dtype):  # noqa: F811
    """Long lists of entries leave less room for rows: narrow tables take the block form of the balance loss, for instance."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(rows + n)
    x, _ = logits_of(gen, rows, n, dtype)
    hosts = hosts_of(gen, rows, n, 256)
    teacher = torch.randn((rows, 256), generator=gen, device="cuda") * 2
    ones, scale = torch.ones(rows, device="cuda"), 512.0 * rows / n
    loss, grad = torch.full((rows,), -7.0, device="cuda"), torch.full((rows, n), 99.0, dtype=x.dtype, device="cuda")
    nb.nbos_policy_distill(x, hosts, teacher, loss, None, ones, 64.0, grad)
    want_l, tol_l, want_g, size = distill64(x, hosts, teacher, 1.0, ones.double() * 64)
    within(loss, want_l, tol_l)
    within(grad, want_g, TOL_P * size + want_g.abs() * (HALF_ULP[dtype] * 1.01) + SMALLEST[dtype])
    even, counts, shares = torch.empty(1, device="cuda"), torch.empty((1, n), dtype=torch.int32, device="cuda"), torch.empty((1, n), device="cuda")
    nb.nbos_policy_balance(x[None], hosts[None], even, counts, shares, None, None, scale, grad[None])
    want = balance64(x, hosts, scale)
    assert torch.equal(counts[0], want[1])
    within(shares[0], want[2], want[2] * (TOL_P + 64 * E) + E * 2.0 ** -100)
    within(even[0], want[0], want[0] * (TOL_P + 64 * E))
    within(grad, want[3], 2 * TOL_P * want[4] + want[3].abs() * (HALF_ULP[dtype] * 1.01) + SMALLEST[dtype])
