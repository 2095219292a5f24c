"""The learned-policy operators against the 64-bit checker.

Tolerances, derived once. Let e = 2^-24 (half an ulp of 32 bits), a = (x - m) / T.
  p_j = 2^((x_j - m) c) / S. The exponent carries three roundings (difference, c, product) of at most 3 e |a| log2(e)
  absolute, so 3 e |a| relative in the power, which itself is good to 2 ulp = 4 e. S is a sum of positive terms
  in which no term goes through more than 32 additions in a lane, 5 over lanes, 8 + 5 over warps and their
  scalings: below 64 e relative. The quotient and scaling add 4 e. Together |dp| <= p (72 + 3 |a|) e. With
  p |a| <= max_t t exp(-t) < 0.4 for the second part and |a| <= 40 where p matters at all: p (72 + 120) e < 200 e p;
  q obeys the same bound. TOL_P = 256 e covers both.
  A loss term q (ln q - ln p) T^2 with |ln q|, |ln p| <= L has error q T^2 (256 e L + 256 e (1 + L)): 512 e (1 + L) T^2.
  A gradient entry g has 256 e (p + q) times its multiplier, and its rounding to the type: half an ulp, 2^-8 |g| in
  bf16 (8 significant bits), 2^-11 |g| in f16 (11) plus half its smallest step 2^-25, and e |g| in f32.
  A share adds the additions over the rows a thread sees, at most `rows` e.
"""
from __future__ import annotations

import math

import numpy as np
import pytest

from oracle import policy as P

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
TOL_P = 256 * E
HALF_ULP = {"float32": E, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
SMALLEST = {"float32": 2.0 ** -126, "bfloat16": 2.0 ** -126, "float16": 2.0 ** -25}
DTYPES = ["float32", "bfloat16", "float16"]
INF = math.inf
# one host; around a warp's and a block's limits, odd sizes, a cluster's rows, rows read twice
SIZES = [(5, 1), (7, 2), (33, 3), (64, 31), (9, 32), (100, 33), (40, 257), (11, 1000), (6, 1024), (5, 1025),
         (4, 4096), (3, 4099), (2, 16385), (2, 32768), (3, 32771), (2, 70001), (1, 262144), (2, 262145),
         (160, 16400), (80, 40001)]


@pytest.fixture(scope="module")
def nb():
    import torch
    from paper_2503_20591_b200 import binding, build as lib_build
    lib_build.build()
    assert torch.cuda.is_available()
    binding.load_library()
    return binding


def make_logits(rng, rows, n, dtype, pad=0, shift=0, spread=2.5, dead=True):
    """A CUDA table whose rows are n + pad apart and start `shift` elements after an allocation's start, some hosts out
    (-inf), one row entirely out; and its values in 64 bits."""
    import torch
    x = rng.normal(size=(rows, n)) * spread
    x[rng.random((rows, n)) < 0.1] = -INF
    if n > 1:
        x[np.arange(rows), rng.integers(0, n, rows)] = 1.0      # never empty by chance
    if dead and rows > 2:
        x[rows // 2] = -INF
    buf = torch.full((rows * (n + pad) + shift,), 99.0, dtype=getattr(torch, dtype), device="cuda")
    t = buf[shift:].view(rows, n + pad)[:, :n]
    t.copy_(torch.from_numpy(x))
    return t, t.double().cpu().numpy()


def make_hosts(rng, rows, n, k):
    h = rng.integers(0, n, size=(rows, k))
    h[rng.random((rows, k)) < 0.15] = -1
    if k > 1 and rows > 1:
        h[0, 1] = h[0, 0]            # listed twice
        h[-1] = -1                   # a row without entries
        h[1, k - 1] = n              # beyond the table
    return h.astype(np.int32)


def close(got, want, tol):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4], got[bad][:4], want[bad][:4],
                           np.broadcast_to(tol, got.shape)[bad][:4])


def distill_bounds(x, hosts, teacher, T, mult, dtype):
    """(tolerance of the loss, tolerance of the gradient) per the module's derivation."""
    loss, grad = P.distill(x, hosts, teacher, T)
    p = np.zeros_like(x)
    depth = np.zeros(len(x))
    for r in range(len(x)):
        p[r], log_p = P._softmax(x[r] / T)
        fin = log_p[np.isfinite(log_p)]
        t = teacher[r][np.isfinite(teacher[r])]
        depth[r] = (np.abs(fin).max() if fin.size else 0) + ((t.max() - t.min()) / T + math.log(len(t)) if t.size else 0)
    q = np.abs(T * p - grad) / T
    g = grad * mult[:, None]
    tol = np.abs(mult)[:, None] * T * TOL_P * (p + q) + np.abs(g) * HALF_ULP[dtype] * 1.01 + SMALLEST[dtype]
    return loss, g, 512 * E * (1 + depth) * T * T, tol


def run_distill(nb, x, hosts, teacher, T, scale, grad_loss=None, in_place=False, grad_pad=0, backward=False):
    import torch
    rows, n = x.shape
    h, t = torch.from_numpy(hosts).cuda(), None if teacher is None else torch.from_numpy(teacher).cuda()
    loss = torch.full((rows,), -7.0, device="cuda")
    stats = torch.full((rows, 2), -7.0, device="cuda")
    gl = None if grad_loss is None else torch.from_numpy(grad_loss).cuda()
    grad = x if in_place else torch.full((rows, n + grad_pad), -7.0, dtype=x.dtype, device="cuda")[:, :n]
    if backward:
        nb.nbos_policy_distill(x, h, t, loss, stats, temperature=T)
        nb.nbos_policy_distill_backward(x, h, t, stats, grad, gl, scale, temperature=T)
    else:
        nb.nbos_policy_distill(x, h, t, loss, stats, gl, scale, grad, temperature=T)
    torch.cuda.synchronize()
    return loss.double().cpu().numpy(), grad.double().cpu().numpy()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,n", SIZES)
def test_distill_matches_the_checker(nb, rows, n, dtype):
    rng = np.random.default_rng(rows * 1000003 + n)
    for k, T, pad, shift in ((3, 1.0, 0, 0), (1, 0.7, 3, 1), (32, 2.0, 8, 0), (70, 1.5, 0, 0)):
        if k == 70 and n > 40000 and dtype != "bfloat16":
            continue
        x, x64 = make_logits(rng, rows, n, dtype, pad, shift)
        hosts = make_hosts(rng, rows, n, k)
        teacher = (rng.normal(size=(rows, k)) * 2).astype(np.float32)
        teacher[rng.random((rows, k)) < 0.05] = -INF
        gl = rng.normal(size=rows).astype(np.float32)
        scale = 64.0
        loss, grad, tol_l, tol_g = distill_bounds(x64, hosts, teacher.astype(np.float64), T, scale * gl.astype(np.float64), dtype)
        got_l, got_g = run_distill(nb, x, hosts, teacher, T, scale, gl, grad_pad=pad)
        close(got_l, loss, tol_l)
        close(got_g, grad, tol_g)
        # the two-call form and the gradient written over the logits give the same
        back_l, back_g = run_distill(nb, x, hosts, teacher, T, scale, gl, backward=True)
        np.testing.assert_array_equal(back_l, got_l)
        close(back_g, grad, tol_g)
        over_l, over_g = run_distill(nb, x, hosts, teacher, T, scale, gl, in_place=True)
        np.testing.assert_array_equal(over_l, got_l)
        np.testing.assert_array_equal(over_g, run_distill_like(nb, x64, dtype, pad, shift, hosts, teacher, T, scale, gl))


def run_distill_like(nb, x64, dtype, pad, shift, hosts, teacher, T, scale, gl):
    """The gradient into a table of the logits' own layout (so that it takes the same path as in place)."""
    import torch
    rows, n = x64.shape

    def table():
        buf = torch.full((rows * (n + pad) + shift,), 99.0, dtype=getattr(torch, dtype), device="cuda")
        return buf[shift:].view(rows, n + pad)[:, :n]

    x, grad = table(), table()
    x.copy_(torch.from_numpy(x64))
    nb.nbos_policy_distill(x, torch.from_numpy(hosts).cuda(), torch.from_numpy(teacher).cuda(), None, None,
                           torch.from_numpy(gl).cuda(), scale, grad, temperature=T)
    return grad.double().cpu().numpy()


def test_distill_teacher_forms(nb):
    """One list of teacher logits for all rows, and none at all (equal)."""
    rng = np.random.default_rng(3)
    x, x64 = make_logits(rng, 50, 100, "float32")
    hosts = make_hosts(rng, 50, 100, 3)
    shared = np.array([0.0, -1.0, -2.5], dtype=np.float32)
    for t, full in ((shared, np.tile(shared, (50, 1))), (None, np.zeros((50, 3), np.float32))):
        loss, grad, tol_l, tol_g = distill_bounds(x64, hosts, full.astype(np.float64), 1.0, np.ones(50), "float32")
        got = run_distill(nb, x, hosts, t, 1.0, 1.0)
        close(got[0], loss, tol_l)
        close(got[1], grad, tol_g)


@pytest.mark.parametrize("n", [48, 3000, 40000])
def test_distill_of_extreme_logits(nb, n):
    """The type's lowest value as a mask, rows of it alone, far apart values, NaN and +inf: no NaN where the formula has
    none, NaN in their own row alone."""
    import torch
    for dtype in DTYPES:
        low = torch.finfo(getattr(torch, dtype)).min
        x = torch.zeros((6, n), dtype=getattr(torch, dtype), device="cuda")
        x[0, 1:] = low           # one host possible
        x[1, :] = low            # all masked alike: an even policy
        x[2, 0] = -low           # far above the others
        x[3, 1] = math.nan
        x[4, 1] = INF
        x[5, 3] = 2.0
        hosts = torch.tensor([[0, 1], [0, 1], [0, 0], [0, 2], [0, 2], [3, 3]], dtype=torch.int32, device="cuda")
        t = torch.tensor([[0.0, -INF]] * 3 + [[0.0, 0.0]] * 3, device="cuda")
        loss, grad = torch.empty(6, device="cuda"), torch.empty_like(x)
        nb.nbos_policy_distill(x, hosts, t, loss, out_grad=grad)
        loss, grad = loss.cpu(), grad.float().cpu()
        assert loss[0] == 0 and not grad[0].any()
        tol = 512 * E * (1 + math.log(n))
        assert abs(loss[1] - math.log(n)) <= tol
        assert abs(float(grad[1, 1]) - 1 / n) <= (HALF_ULP[dtype] * 1.01 + TOL_P) / n + SMALLEST[dtype]
        assert loss[2] == 0 and not grad[2].any()
        for r in (3, 4):
            assert torch.isnan(loss[r]) and torch.isnan(grad[r]).all()
        assert not torch.isnan(loss[5]) and not torch.isnan(grad[5]).any()


def test_distill_gradient_is_the_slope(nb):
    """Central differences with h = 1/64: the third derivative of the loss in one logit is at most T^-1 / 6 * T^... <= 1 for
    T = 1, so h^2 / 6 < 5e-5, and the two losses' errors give 2 tol / (2 h) = 64 tol."""
    rng = np.random.default_rng(8)
    x, x64 = make_logits(rng, 6, 40, "float32", dead=False)
    hosts = make_hosts(rng, 6, 40, 3)
    teacher = rng.normal(size=(6, 3)).astype(np.float32)
    _, _, tol_l, _ = distill_bounds(x64, hosts, teacher.astype(np.float64), 1.0, np.ones(6), "float32")
    grad = run_distill(nb, x, hosts, teacher, 1.0, 1.0)[1]
    h = 1 / 64
    for j in range(0, 40, 3):
        up, down = x.clone(), x.clone()
        up[:, j] += h
        down[:, j] -= h
        slope = (run_distill(nb, up, hosts, teacher, 1.0, 1.0)[0] - run_distill(nb, down, hosts, teacher, 1.0, 1.0)[0]) / (2 * h)
        close(grad[:, j], slope, h * h / 6 + 64 * tol_l + 2 * E)


# ---- balance --------------------------------------------------------------------------------------------------------
def run_balance(nb, x, hosts, scale=1.0, grad_loss=None, grad=None, backward=False):
    import torch
    groups = x.shape[0]
    n = x.shape[2]
    h = torch.from_numpy(hosts).cuda()
    loss = torch.full((groups,), -7.0, device="cuda")
    counts = torch.full((groups, n), -7, dtype=torch.int32, device="cuda")
    shares = torch.full((groups, n), -7.0, device="cuda")
    stats = torch.full((groups, x.shape[1], 2), -7.0, device="cuda")
    gl = None if grad_loss is None else torch.from_numpy(grad_loss).cuda()
    grad = torch.full(x.shape, -7.0, dtype=x.dtype, device="cuda") if grad is None else grad
    if backward:
        nb.nbos_policy_balance(x, h, loss, counts, shares, stats)
        nb.nbos_policy_balance_backward(x, h, stats, grad, gl, scale)
    else:
        nb.nbos_policy_balance(x, h, loss, counts, shares, stats, gl, scale, grad)
    torch.cuda.synchronize()
    return tuple(v.cpu().numpy() if v.dtype == torch.int32 else v.double().cpu().numpy() for v in (loss, counts, shares, grad))


def check_balance(nb, x, x64, hosts, scale, gl, dtype, **kw):
    groups, rows, n = x64.shape
    loss, counts, shares, grad = run_balance(nb, x, hosts, scale, gl, **kw)
    for g in range(groups):
        want = P.balance(x64[g], hosts[g])
        np.testing.assert_array_equal(counts[g], want[1])
        rel = TOL_P + rows * E
        close(shares[g], want[2], want[2] * rel + E * 2.0 ** -100)
        close(loss[g], want[0], want[0] * rel)
        live = ((hosts[g] >= 0) & (hosts[g] < n)).any(1)
        f = want[1] / max(1, want[1].sum())
        p = np.stack([P._softmax(r)[0] for r in x64[g]]) * live[:, None]
        mult = scale * float(gl[g])
        exact = want[3] * mult
        # p (f - f.p): twice the error of p on either part
        tol = abs(mult) * n / max(1, live.sum()) * p * (f + p @ f[:, None]) * 2 * TOL_P
        close(grad[g], exact, tol + np.abs(exact) * HALF_ULP[dtype] * 1.01 + SMALLEST[dtype])
    return loss, counts, shares, grad


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("groups,rows,n", [(1, 5, 1), (3, 7, 2), (2, 33, 3), (1, 640, 31), (5, 90, 32), (1, 1500, 33), (4, 40, 257),
                                           (2, 11, 1000), (3, 60, 1024), (1, 300, 1025), (2, 40, 4096), (1, 9, 4099),
                                           (2, 3, 16385), (1, 4, 32771), (1, 160, 16400), (2, 40, 40001), (1, 3, 131072), (1, 3, 131073), (300, 2, 40)])
def test_balance_matches_the_checker(nb, groups, rows, n, dtype):
    rng = np.random.default_rng(groups * 7919 + rows * 104729 + n)
    for k, pad, shift in ((3, 0, 0), (1, 3, 1), (40, 8, 0)):
        x2, x64 = make_logits(rng, groups * rows, n, dtype, pad, shift)
        x = x2.unflatten(0, (groups, rows))
        x64 = x64.reshape(groups, rows, n)
        hosts = np.stack([make_hosts(rng, rows, n, k) for _ in range(groups)])
        if groups > 2:
            hosts[1] = -1             # a group without a choice
        gl = rng.normal(size=groups).astype(np.float32)
        scale = 512.0 * rows / n
        fused = check_balance(nb, x, x64, hosts, scale, gl, dtype)
        again = run_balance(nb, x, hosts, scale, gl)
        for a, b in zip(fused, again):
            np.testing.assert_array_equal(a, b)          # no order that changes from run to run
        check_balance(nb, x, x64, hosts, scale, gl, dtype, backward=True)
        check_balance(nb, x, x64, hosts, scale, gl, dtype, grad=x)   # over the logits, last


def test_balance_counts_of_many_rows_and_hosts(nb):
    """More hosts than counters fit in shared memory; every choice the same host; ids beyond the table."""
    import torch
    rng = np.random.default_rng(5)
    for rows, n, k in ((20000, 9000, 4), (70001, 8192, 2), (50000, 64, 8)):
        hosts = rng.integers(-1, n + 1, size=(1, rows, k)).astype(np.int32)
        hosts[0, : rows // 3] = n - 1
        x = torch.zeros((1, rows, n), dtype=torch.bfloat16, device="cuda")
        loss, counts, shares, grad = run_balance(nb, x, hosts)
        np.testing.assert_array_equal(counts[0], np.bincount(hosts[(hosts >= 0) & (hosts < n)], minlength=n))
        close(shares[0], np.full(n, 1 / n), (TOL_P + rows * E) / n)
        close(loss, np.ones(1), TOL_P + rows * E)


@pytest.mark.parametrize("n", [48, 3000, 140000])
def test_balance_of_extreme_logits(nb, n):
    import torch
    for dtype in DTYPES:
        low = torch.finfo(getattr(torch, dtype)).min
        x = torch.zeros((2, 5, n), dtype=getattr(torch, dtype), device="cuda")
        x[0, 0, 1:] = low
        x[0, 1, :] = low
        x[0, 2, :] = -INF
        x[0, 3, 0] = -low
        x[0, 4] = math.nan        # its row has no choice: left out altogether
        x[1, 2, 1] = math.nan     # a live row: its group's loss and shares and its own gradient
        hosts = np.zeros((2, 5, 2), np.int32)
        hosts[0, 4] = -1
        loss, counts, shares, grad = run_balance(nb, x, hosts, 64.0)
        # shares of host 0: one, 1 / n, nothing, one, of four live rows
        want = (2 + 1 / n) / 4
        assert abs(shares[0, 0] - want) <= want * 2 * TOL_P
        assert abs(loss[0] - n * want) <= n * want * 2 * TOL_P
        assert np.isfinite(grad[0]).all() and not grad[0, 4].any() and not grad[0, 2].any()
        assert counts[0].sum() == 8 and counts[1, 0] == 10
        assert np.isnan(loss[1]) and np.isnan(shares[1]).all()
        assert np.isnan(grad[1, 2]).all() and np.isfinite(np.delete(grad[1], 2, 0)).all()


def test_balance_gradient_is_the_slope(nb):
    """As for distillation: h = 1/64, third derivative at most n / live, error of a loss TOL_P + rows e."""
    import torch
    rng = np.random.default_rng(9)
    x2, _ = make_logits(rng, 6, 20, "float32", dead=False)
    x = x2.view(1, 6, 20)
    hosts = make_hosts(rng, 6, 20, 3)[None]
    loss, _, _, grad = run_balance(nb, x, hosts)
    h, live = 1 / 64, 5
    for r in range(6):
        for j in range(0, 20, 5):
            up, down = x.clone(), x.clone()
            up[0, r, j] += h
            down[0, r, j] -= h
            slope = (run_balance(nb, up, hosts)[0] - run_balance(nb, down, hosts)[0]) / (2 * h)
            close(grad[0, r, j], slope[0], h * h / 6 * 20 / live + 64 * loss[0] * (TOL_P + 6 * E))


# ---- sampling -------------------------------------------------------------------------------------------------------
def run_sample(nb, x, u, **kw):
    import torch
    rows, draws = u.shape
    hosts = torch.full((rows, draws), -9, dtype=torch.int32, device="cuda")
    found = torch.full((rows,), -9, dtype=torch.int32, device="cuda")
    kw = {k: None if v is None else torch.from_numpy(np.ascontiguousarray(v)).cuda() for k, v in kw.items()}
    nb.nbos_policy_sample(x, torch.from_numpy(u).cuda(), hosts, found, **kw)
    torch.cuda.synchronize()
    return hosts.cpu().numpy(), found.cpu().numpy()


def settings(rng, rows, n, exact):
    """Per-row filters: each off for some rows, at its ends for others."""
    T = np.full(rows, P_ONE, np.float32) if exact else rng.uniform(0.3, 2.0, rows).astype(np.float32)
    T[rng.random(rows) < 0.1] = rng.choice([0.0, -1.0, math.nan, 2.0 ** -20])
    k = rng.choice([-1, 0, 1, 2, 3, 7, 50, n - 1, n, n + 5], rows).astype(np.int32)
    p = rng.choice([-0.5, 0.0, 1e-7, 0.1, 0.5, 0.9, 0.99, 0.9999999, 1.0, 2.0, math.nan], rows).astype(np.float32)
    q = rng.choice([-1.0, 0.0, math.nan, 1e-6, 0.01, 0.125, 0.5, 1.0, 3.0], rows).astype(np.float32)
    return T, k, p, q


P_ONE = np.float32(1.4426950408889634)   # c = 1: whole logits have exact weights, many of them equal


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,n", [(40, 1), (60, 2), (80, 31), (80, 32), (80, 100), (60, 257), (40, 1000), (40, 1024), (24, 1025),
                                    (16, 4099), (8, 20000)])
def test_sample_matches_the_checker_exactly(nb, rows, n, dtype):
    """Whole logits at c = 1: weights are powers of two, so the checker's are the library's and every host must agree;
    nearly every cut falls into ties."""
    import torch
    rng = np.random.default_rng(rows * 31 + n)
    for draws, pad, shift, depth in ((1, 0, 0, 4), (3, 3, 1, 12), (8, 8, 0, 40)):
        v = -rng.integers(0, depth, size=(rows, n)).astype(np.float64) + rng.integers(-30, 30, size=(rows, 1))
        v[rng.random((rows, n)) < 0.1] = -INF
        v[rng.random((rows, n)) < 0.02] = math.nan
        v[v == 0] = rng.choice([0.0, -0.0], int((v == 0).sum()))     # equal logits, whatever their sign
        v[0] = -INF
        buf = torch.full((rows * (n + pad) + shift,), 99.0, dtype=getattr(torch, dtype), device="cuda")
        x = buf[shift:].view(rows, n + pad)[:, :n]
        x.copy_(torch.from_numpy(v))
        u = rng.random((rows, draws)).astype(np.float32)
        u[rng.random((rows, draws)) < 0.1] = rng.choice([0.0, 1.0, -1.0, 2.0, math.nan, 1 - 2.0 ** -24])
        T, k, p, q = settings(rng, rows, n, exact=True)
        for kw in (dict(temperature=T), dict(temperature=T, top_k=k), dict(temperature=T, top_p=p), dict(temperature=T, min_p=q),
                   dict(temperature=T, top_k=k, top_p=p, min_p=q)):
            got = run_sample(nb, x, u, **kw)
            want = P.sample(x.float().cpu().numpy(), u, **kw)
            np.testing.assert_array_equal(got[0], want[0])
            np.testing.assert_array_equal(got[1], want[1])


def torch_sample(x, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """The definition in torch operations on the GPU: the same 32-bit powers, sums in 64-bit integers."""
    import torch
    rows, n = x.shape
    x = x.float()
    x = torch.where(torch.isnan(x), -INF, x).clamp(max=3.402823466e38)
    m = x.amax(1, keepdim=True)
    T = torch.ones((rows, 1), device="cuda") if temperature is None else torch.from_numpy(temperature).cuda()[:, None]
    greedy = ~(T > 2.0 ** -20)
    T = torch.where(greedy, 1.0, T)
    w = (torch.exp2((x - torch.where(m > -INF, m, 0.0)) * (torch.full_like(T, 1.4426950408889634) / T)) * 2.0 ** 31).long()
    xs, order = x.sort(dim=1, descending=True, stable=True)
    w = w.gather(1, order)
    place = torch.arange(n, device="cuda")
    w *= ~greedy | (place == 0)
    if top_k is not None:
        k = torch.from_numpy(top_k).cuda()[:, None]
        w *= (place < k) | (k <= 0)

    def part(total, steps):
        return steps * (total >> 24) + ((steps * (total & 0xFFFFFF)) >> 24)

    stays = torch.ones_like(w, dtype=torch.bool)
    if top_p is not None:
        p = torch.from_numpy(top_p).cuda()[:, None]
        steps = (torch.nan_to_num(p, 1.0).clamp(0, 1) * 2 ** 24).long()
        stays &= (w.cumsum(1) - w < part(w.sum(1, keepdim=True), steps).clamp(min=1)) | ~(p < 1)
    if min_p is not None:
        q = torch.from_numpy(min_p).cuda()[:, None]
        stays &= (w >= (torch.nan_to_num(q, 0.0).clamp(0, 1) * 2.0 ** 31).long())
    w = torch.empty_like(w).scatter_(1, order, w * stays)
    out = []
    steps = (torch.nan_to_num(torch.from_numpy(u).cuda(), 0.0).clamp(0, 1) * 2 ** 24).long().clamp(max=2 ** 24 - 1)
    for d in range(u.shape[1]):
        run = w.cumsum(1)
        h = (run <= part(run[:, -1:], steps[:, d:d + 1])).sum(1, keepdim=True)
        h = torch.where(run[:, -1:] > 0, h, -1)
        out.append(h)
        w.scatter_(1, h.clamp(min=0), 0)
    hosts = torch.cat(out, 1).int()
    return hosts.cpu().numpy(), (hosts >= 0).sum(1).int().cpu().numpy()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,n", [(3000, 32), (2000, 250), (900, 1000), (900, 1024), (300, 1500), (200, 4096), (100, 8191), (9, 32768),
                                    (5, 32769), (1, 65536), (3, 100001), (2, 262144), (2, 262145), (1, 1 << 20)])
def test_sample_matches_the_definition_on_real_logits(nb, rows, n, dtype):
    rng = np.random.default_rng(rows + n)
    x, _ = make_logits(rng, rows, n, dtype)
    u = rng.random((rows, 3)).astype(np.float32)
    T, k, p, q = settings(rng, rows, n, exact=False)
    for kw in (dict(), dict(temperature=T), dict(top_k=k), dict(top_p=p, temperature=T), dict(temperature=T, top_k=k, top_p=p, min_p=q)):
        got = run_sample(nb, x, u, **kw)
        want = torch_sample(x, u, **kw)
        np.testing.assert_array_equal(got[0], want[0])
        np.testing.assert_array_equal(got[1], want[1])


def test_sample_follows_the_distribution(nb):
    """200,000 draws from one row: each host's frequency within 6 standard deviations of softmax, in 64 bits."""
    import torch
    rng = np.random.default_rng(4)
    row = rng.normal(size=50) * 2
    draws = 200_000
    x = torch.from_numpy(np.tile(row, (draws, 1))).float().cuda()
    hosts, found = run_sample(nb, x, rng.random((draws, 1)).astype(np.float32), temperature=np.full(draws, 1.3, np.float32))
    p = P._softmax(x[0].double().cpu().numpy() / 1.3)[0]
    freq = np.bincount(hosts[:, 0], minlength=50) / draws
    close(freq, p, 6 * np.sqrt(p * (1 - p) / draws) + 1e-5)
    assert (found == 1).all()


def test_sample_of_extreme_logits(nb):
    import torch
    for dtype in DTYPES:
        info = torch.finfo(getattr(torch, dtype))
        for n in (40, 3000, 40000):
            x = torch.zeros((6, n), dtype=getattr(torch, dtype), device="cuda")
            x[0] = -INF
            x[1] = math.nan
            x[2] = info.min
            x[3, n - 1] = INF
            x[4] = info.min
            x[4, 7] = info.max
            x[5, 2:] = -INF
            u = np.full((6, 3), 0.5, np.float32)
            hosts, found = run_sample(nb, x, u, top_p=np.full(6, 0.9, np.float32), top_k=np.full(6, n - 1, np.int32))
            assert hosts[0].tolist() == [-1] * 3 == hosts[1].tolist() and found[0] == found[1] == 0
            assert found[2] == 3 and len(set(hosts[2].tolist())) == 3
            assert hosts[4].tolist() == [7, -1, -1] and found[4] == 1
            assert sorted(hosts[5].tolist()) == [-1, 0, 1] and found[5] == 2
            assert hosts[3].tolist() == [n - 1, -1, -1] and found[3] == 1


# ---- the entry points in use ----------------------------------------------------------------------------------------
def test_empty_batches(nb):
    import torch
    x = torch.empty((0, 16), device="cuda")
    nb.nbos_policy_distill(x, torch.empty((0, 3), dtype=torch.int32, device="cuda"), None, torch.empty(0, device="cuda"))
    nb.nbos_policy_sample(x, torch.empty((0, 3), device="cuda"), torch.empty((0, 3), dtype=torch.int32, device="cuda"))
    loss, counts = torch.full((2,), 9.0, device="cuda"), torch.full((2, 16), 9, dtype=torch.int32, device="cuda")
    shares = torch.full((2, 16), 9.0, device="cuda")
    nb.nbos_policy_balance(torch.empty((2, 0, 16), device="cuda"), torch.empty((2, 0, 3), dtype=torch.int32, device="cuda"),
                           loss, counts, shares)
    assert not loss.any() and not counts.any() and not shares.any()


def test_wrong_tensors_are_refused(nb):
    import torch
    x, h = torch.zeros((4, 8), device="cuda"), torch.zeros((4, 3), dtype=torch.int32, device="cuda")
    loss = torch.zeros(4, device="cuda")
    bad = [
        (TypeError, lambda: nb.nbos_policy_distill(x, h.long(), None, loss)),
        (ValueError, lambda: nb.nbos_policy_distill(x, h[:3], None, loss)),
        (ValueError, lambda: nb.nbos_policy_distill(x.t(), h, None, loss)),
        (ValueError, lambda: nb.nbos_policy_distill(x, h, None, loss[:3])),
        (ValueError, lambda: nb.nbos_policy_distill(x, h, torch.zeros(4, device="cuda"), loss)),
        (ValueError, lambda: nb.nbos_policy_distill(x, h, None, loss, out_grad=x.half())),
        (ValueError, lambda: nb.nbos_policy_distill(x, h, None, loss.cpu())),
        (ValueError, lambda: nb.nbos_policy_distill(x, h.t().contiguous().t(), None, loss)),
        (ValueError, lambda: nb.nbos_policy_balance(x, h, loss, h)),
        (ValueError, lambda: nb.nbos_policy_sample(x, torch.zeros((3, 1), device="cuda"), h)),
        (TypeError, lambda: nb.nbos_policy_sample(x, torch.zeros((4, 3), device="cuda"), h, top_k=loss)),
        (ValueError, lambda: nb.nbos_policy_sample(x, torch.zeros((4, 3), device="cuda"), h, top_p=loss[:2])),
        (nb.NbosError, lambda: nb.nbos_policy_distill(x, h, None, loss, temperature=0.0)),
        (nb.NbosError, lambda: nb.nbos_policy_sample(x, torch.zeros((4, 9), device="cuda"),
                                                     torch.zeros((4, 9), dtype=torch.int32, device="cuda"))),
    ]
    for kind, call in bad:
        with pytest.raises(kind):
            call()


def test_autograd(nb):
    """policy.distill_loss and balance_loss under autograd against the checker's gradients, in a table with strides."""
    import torch
    from paper_2503_20591_b200 import policy
    rng = np.random.default_rng(12)
    x2, x64 = make_logits(rng, 60, 37, "float32", pad=2)
    x = x2.unflatten(0, (3, 20)).detach().requires_grad_(True)
    hosts = np.stack([make_hosts(rng, 20, 37, 3) for _ in range(3)])
    teacher = rng.normal(size=(3, 20, 3)).astype(np.float32)
    h, t = torch.from_numpy(hosts).cuda(), torch.from_numpy(teacher).cuda()
    loss = policy.distill_loss(x, h, t, temperature=2.0)
    even, counts, shares = policy.balance_loss(x, h)
    assert loss.shape == (3, 20) and even.shape == (3,) and counts.shape == shares.shape == (3, 37)
    (loss.mean() + 0.01 * even.sum()).backward()
    _, g1, _, tol1 = distill_bounds(x64, hosts.reshape(60, 3), teacher.reshape(60, 3).astype(np.float64), 2.0,
                                    np.full(60, 1 / 60), "float32")
    g2 = np.concatenate([P.balance(x64.reshape(3, 20, 37)[g], hosts[g])[3] for g in range(3)]) * 0.01
    close(x.grad.double().cpu().numpy().reshape(60, 37), g1 + g2, tol1 + 0.01 * 37 / 10 * 4 * TOL_P + 4 * E * (np.abs(g1) + np.abs(g2)))


def test_other_streams_and_graphs(nb):
    """Work on a stream of the caller's, and the calls captured into a graph and replayed on new inputs."""
    import torch
    rng = np.random.default_rng(13)
    stream = torch.cuda.Stream()
    x = torch.empty((1, 500, 200), device="cuda")
    hosts = torch.empty((1, 500, 3), dtype=torch.int32, device="cuda")
    u = torch.rand((1, 500, 3), device="cuda")
    loss, even = torch.empty((1, 500), device="cuda"), torch.empty(1, device="cuda")
    counts = torch.empty((1, 200), dtype=torch.int32, device="cuda")
    grad = torch.empty_like(x)
    drawn = torch.empty_like(hosts)

    def fill(seed):
        r = np.random.default_rng(seed)
        x.copy_(torch.from_numpy(r.normal(size=x.shape)))
        hosts.copy_(torch.from_numpy(make_hosts(r, 500, 200, 3)[None]))

    def calls():
        nb.nbos_policy_distill(x, hosts, None, loss, out_grad=grad, stream=stream)
        nb.nbos_policy_balance(x, hosts, even, counts, stream=stream)
        nb.nbos_policy_sample(x, u, drawn, stream=stream)

    fill(1)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        calls()
    stream.synchronize()
    first = [v.clone() for v in (loss, even, counts, grad, drawn)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        calls()
    fill(2)
    graph.replay()
    torch.cuda.synchronize()
    second = [v.clone() for v in (loss, even, counts, grad, drawn)]
    assert not torch.equal(first[0], second[0])
    fill(1)
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(first, (loss, even, counts, grad, drawn)):
        assert torch.equal(a, b)


def test_offsets_beyond_31_bits(nb):
    """Rows that start past 2^31 elements: the last row must answer as the same row alone."""
    import torch
    n, rows = 65536, 33000
    x = torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda")
    x[-1] = torch.randn(n, device="cuda")
    hosts = torch.randint(0, n, (rows, 3), dtype=torch.int32, device="cuda")
    u = torch.rand((rows, 3), device="cuda")
    loss, grad = torch.empty(rows, device="cuda"), torch.empty_like(x)
    nb.nbos_policy_distill(x, hosts, None, loss, out_grad=grad)
    one_loss, one_grad = torch.empty(1, device="cuda"), torch.empty_like(x[-1:])
    nb.nbos_policy_distill(x[-1:], hosts[-1:], None, one_loss, out_grad=one_grad)
    torch.testing.assert_close(loss[-1:], one_loss, rtol=64 * TOL_P, atol=0)
    torch.testing.assert_close(grad[-1:], one_grad, rtol=2.0 ** -7, atol=2.0 ** -30)
    drawn, one = torch.empty((rows, 3), dtype=torch.int32, device="cuda"), torch.empty((1, 3), dtype=torch.int32, device="cuda")
    nb.nbos_policy_sample(x, u, drawn)
    nb.nbos_policy_sample(x[-1:].contiguous(), u[-1:].contiguous(), one)
    assert torch.equal(drawn[-1:], one)
    even, counts = torch.empty(1, device="cuda"), torch.empty((1, n), dtype=torch.int32, device="cuda")
    nb.nbos_policy_balance(x, hosts, even, counts, out_grad=grad)
    assert int(counts.sum()) == 3 * rows and abs(float(even) - 1.0) < 0.05 and bool(torch.isfinite(grad[-1]).all())


def test_a_policy_learns_the_rule(nb):
    """The operators together: a small policy trained on the exact rule's hosts comes to choose them, and what it samples is
    feasible and distinct."""
    from paper_2503_20591_b200 import train_policy
    result = train_policy.train(hosts=64, snapshots=8, batch=256, steps=120, report=lambda text: None)
    first, last = result["history"][0], result["history"][-1]
    assert last[0] < 0.6 * first[0] and last[2] > first[2]
    assert result["feasible"] and result["distinct"] and 0 < result["found"] <= 3
