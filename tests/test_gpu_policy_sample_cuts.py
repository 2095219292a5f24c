"""Sampling where a cut falls on logits that are hard to tell apart: hosts drawn must be those of the definition, exactly, in every form
of the kernel (a warp's registers, one warp, a block, a cluster, rows kept in the workspace)."""
from __future__ import annotations

import math

import numpy as np
import pytest

from oracle import policy as P
from test_gpu_policy import nb, run_sample, torch_sample  # noqa: F401 (nb is a fixture)

pytestmark = pytest.mark.gpu
INF = math.inf

FORMS = [(60, 100), (60, 300), (40, 1024), (1200, 1500), (1200, 4096), (30, 3000), (12, 8191), (4, 40000), (2, 262145)]


def same(got, want):
    np.testing.assert_array_equal(got[0], want[0])
    np.testing.assert_array_equal(got[1], want[1])


def table(v, dtype):
    import torch
    return torch.from_numpy(v).to("cuda", getattr(torch, dtype))


def top_ks(rng, rows, n):
    return rng.choice([50, 110, 130, n // 3, n // 2, n - 1], rows).astype(np.int32)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,n", FORMS)
def test_top_k_cut_at_zero(nb, rows, n, dtype):  # noqa: F811
    """Scores of which many are 0: half or a tenth of the hosts above it, a few alone, zeros of both signs, zeros as the lowest score."""
    rng = np.random.default_rng(rows * 7 + n)
    normal = rng.normal(size=(rows, n))
    few = np.where(rng.random((rows, n)) < 20 / n, rng.random((rows, n)) + 0.1, 0.0)
    signed = np.where(rng.random((rows, n)) < 0.5, rng.choice([0.0, -0.0], (rows, n)), np.maximum(normal - 1, 0))
    out = rng.random((rows, n)) < 0.2
    for v in (np.maximum(normal, 0), np.maximum(normal - 1.3, 0) * 3, few, signed, np.where(out, -INF, np.maximum(normal - 1, 0)),
              np.where(out, -1.0, np.maximum(normal - 1, 0))):
        x = table(v, dtype)
        u = rng.random((rows, 8)).astype(np.float32)
        k = top_ks(rng, rows, n)
        p = rng.choice([0.5, 0.9, 0.99, 1.0], rows).astype(np.float32)
        for kw in (dict(top_k=k), dict(top_k=k, top_p=p)):
            same(run_sample(nb, x, u, **kw), torch_sample(x, u, **kw))


@pytest.mark.parametrize("rows,n", [(60, 300), (40, 1024), (10, 3000)])
def test_whole_scores_of_which_many_are_zero(nb, rows, n):  # noqa: F811
    """The same against the oracle: whole logits at c = 1 have exact weights."""
    rng = np.random.default_rng(n)
    v = np.maximum(rng.integers(-9, 6, size=(rows, n)), 0).astype(np.float32)
    v[: rows // 2] = np.where(rng.random((rows // 2, n)) < 20 / n, v[: rows // 2], 0)
    u = rng.random((rows, 8)).astype(np.float32)
    kw = dict(temperature=np.full(rows, np.float32(1.4426950408889634)), top_k=top_ks(rng, rows, n))
    same(run_sample(nb, table(v, "float32"), u, **kw), P.sample(v, u, **kw))


LOG2E = np.float32(1.4426950408889634)


def near_the_best(rng, rows, n, best, below, some=40):
    """Rows in which `some` hosts or so have `best`, many `below` (its neighbour in 32 bits), others half of it or nothing."""
    v = np.full((rows, n), best / 2, np.float32)
    v[rng.random((rows, n)) < 0.6] = below
    v[rng.random((rows, n)) < 0.1] = -INF
    v[rng.random((rows, n)) < some / n] = best
    v[:, n // 2] = best
    return v


@pytest.mark.parametrize("rows,n", FORMS[1:])
@pytest.mark.parametrize("best,c", [(2.0 ** 28, 1.0), (400.0, 2.0 ** 20)])
def test_top_k_where_the_next_value_has_no_weight(nb, rows, n, best, c):  # noqa: F811
    """One step of 32 bits below the best logit is 32 powers of two: nothing but the best has a weight."""
    rng = np.random.default_rng(rows + n)
    T = np.float32(LOG2E / np.float32(c))
    assert LOG2E / T == c
    below = np.nextafter(np.float32(best), np.float32(0))
    assert (np.float32(best) - below) * c in (16, 32)       # 2^28 is a power of two: half a step below it
    if (np.float32(best) - below) * c == 16:
        best, below = best + 32, best
    v = near_the_best(rng, rows, n, best, below)
    u = rng.random((rows, 8)).astype(np.float32)
    for k in (50, 120, n - 1):
        kw = dict(temperature=np.full(rows, T), top_k=np.full(rows, k, np.int32))
        got, want = run_sample(nb, table(v, "float32"), u, **kw), torch_sample(table(v, "float32"), u, **kw)
        same(got, want)
        assert (got[1] > 0).all()


@pytest.mark.parametrize("rows,n", FORMS)
@pytest.mark.parametrize("best,c", [(2.0 ** 27 + 16, 1.5), (400.0, 1.5 * 2.0 ** 19), (200.0, 0.0)])
def test_top_k_where_the_next_value_has_a_weight(nb, rows, n, best, c):  # noqa: F811
    """One step of 32 bits below the best logit is 24 powers of two (22 at 200 with T = 1e-6): its hosts come after the best ones."""
    rng = np.random.default_rng(rows + n)
    T = np.float32(LOG2E / np.float32(c)) if c else np.float32(1e-6)
    below = np.nextafter(np.float32(best), np.float32(0))
    if c:
        assert LOG2E / T == np.float32(c) and (np.float32(best) - below) * c == 24
    v = near_the_best(rng, rows, n, best, below, some=3)
    u = rng.random((rows, 8)).astype(np.float32)
    for k in (20, 50, 120, n - 1):
        kw = dict(temperature=np.full(rows, T), top_k=np.full(rows, k, np.int32))
        got, want = run_sample(nb, table(v, "float32"), u, **kw), torch_sample(table(v, "float32"), u, **kw)
        same(got, want)
        assert (got[1] == 8).all()
