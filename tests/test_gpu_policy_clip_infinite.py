"""Clipping by an infinite max_norm clips nothing, whatever the values are; and what clipping does to a training step."""
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


@pytest.mark.parametrize("kind", ["2", "inf"])
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("sizes", [(7, 300), (5, 3_000_001)])   # one cluster, two launches
def test_an_infinite_bound_leaves_infinite_values_alone(nb, sizes, in_place, kind):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    tensors = [torch.randn(n, generator=gen, device="cuda").to(t) for n, t in zip(sizes, (torch.float32, torch.bfloat16))]
    for odd in (INF, -INF):
        for t in tensors:
            t[2] = odd
            before = [x.clone() for x in tensors]
            outs = tensors if in_place else [torch.full_like(x, -7) for x in tensors]
            norm = torch.empty((), device="cuda")
            nb.nbos_policy_clip(tensors, INF, norm, outs, norm_kind=nb.NBOS_NORM_2 if kind == "2" else nb.NBOS_NORM_INF)
            assert float(norm) == INF
            assert all(torch.equal(x, y) for x, y in zip(outs, before))
            t[2] = 1.0
    # a finite bound: as the formula says
    tensors[0][2] = INF
    norm, outs = torch.empty((), device="cuda"), [torch.empty_like(x) for x in tensors]
    nb.nbos_policy_clip(tensors, 1.0, norm, outs)
    assert float(norm) == INF and outs[0][2].isnan() and (outs[1] == 0).all() and int(outs[0].count_nonzero()) == 1
    # a NaN spoils everything at any bound
    tensors[0][2] = math.nan
    nb.nbos_policy_clip(tensors, INF, norm, outs)
    assert norm.isnan() and all(x.isnan().all() for x in outs)


def test_measuring_the_norm_of_a_step_that_overflowed(nb):
    import torch
    from paper_2503_20591_b200 import policy
    p = torch.nn.Parameter(torch.zeros(1000, device="cuda"))
    p.grad = torch.arange(1000, device="cuda").float()
    p.grad[17] = INF
    want = p.grad.clone()
    assert float(policy.clip_gradients([p], INF)) == INF
    assert torch.equal(p.grad, want)


@pytest.mark.parametrize("table,max_norm", [(True, 0.05), (False, 0.05), (False, 1e6)])
def test_a_training_step_is_clipped(nb, monkeypatch, table, max_norm):
    """After each call the gradients that the optimizer sees have the norm min(norm, max_norm): within the factor's rounding and a value's
    (2^-24 each) and the 1e-6 beside the norm."""
    import torch
    from paper_2503_20591_b200 import policy, train_policy
    seen, clip = [], policy.clip_gradients

    def watched(parameters, bound, *args):
        parameters = list(parameters)
        total = lambda: float(sum(p.grad.double().square().sum() for p in parameters if p.grad is not None).sqrt())
        before = total()
        norm = clip(parameters, bound, *args)
        seen.append((before, float(norm), total()))
        return norm

    monkeypatch.setattr(policy, "clip_gradients", watched)
    train_policy.train(hosts=64, snapshots=3, batch=100, steps=4, report=lambda text: None, blocks=1, max_norm=max_norm, table=table)
    assert len(seen) == 4
    for before, norm, after in seen:
        assert abs(norm - before) <= 2.0 ** -20 * before
        assert abs(after - min(before, max_norm)) <= 2.0 ** -20 * after + 1e-6 * max_norm / before
    assert any(before > max_norm for before, *_ in seen) == (max_norm < 1)
