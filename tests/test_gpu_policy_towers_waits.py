"""A wait that runs out in a two-tower kernel: its blocks leave, the outputs are marked, the status says so once, and the next call is
right. The waits run out because a launch is told to copy nothing, with a limit of 2 ms."""
from __future__ import annotations

import pytest

from test_gpu_policy_towers import make, nb   # noqa: F401 (nb is a fixture)

pytestmark = pytest.mark.gpu

SCORES, GRADIENT, REQUESTS, HOSTS = range(4)
SIZES = [(1, 300, 5000, 64, False, 3), (2, 700, 260, 300, True, 9), (1, 20, 900, 40, True, 1)]


def forward(nb, c):
    import torch
    shape, k = c["hosts"].shape[:-1], c["hosts"].shape[-1]
    loss, stats = torch.full(shape, -7.0, device="cuda"), torch.empty((*shape, 2 + k), device="cuda")
    nb.nbos_policy_towers(c["requests"], c["host_vectors"], c["hosts"], c["teacher_logits"], loss, stats, asks=c["asks"], room=c["room"])
    return loss, stats


def backward(nb, c, stats):
    import torch
    grads = [torch.full(c[n].shape, -7.0, dtype=c[n].dtype, device="cuda") for n in ("requests", "host_vectors")]
    nb.nbos_policy_towers_backward(c["requests"], c["host_vectors"], c["hosts"], c["teacher_logits"], stats, *grads, asks=c["asks"], room=c["room"])
    return grads


@pytest.mark.parametrize("groups,rows,hosts,width,mask,k", SIZES)
@pytest.mark.parametrize("kernel", [SCORES, GRADIENT, REQUESTS, HOSTS])
def test_a_wait_that_runs_out(nb, kernel, groups, rows, hosts, width, mask, k):
    import torch
    c = make(groups, rows, hosts, width, k, "bfloat16", mask, 7)
    loss, stats = forward(nb, c)
    grads = backward(nb, c, stats)
    assert nb.nbos_policy_towers_status() == nb.NBOS_OK
    nb.nbos_probe_towers_stall(kernel, 2_000_000)
    if kernel == SCORES:
        assert forward(nb, c)[0].isnan().all()
    else:
        got = backward(nb, c, stats)
        assert torch.equal(got[0], grads[0]) if kernel == HOSTS else got[0].isnan().all()
        assert got[1].isnan().all()
    # until the status is asked, all that follows is marked
    assert forward(nb, c)[0].isnan().all()
    assert all(g.isnan().all() for g in backward(nb, c, stats))
    assert nb.nbos_policy_towers_status() == nb.NBOS_ERR_DEVICE_TIMEOUT
    assert nb.nbos_policy_towers_status() == nb.NBOS_OK
    again, saved = forward(nb, c)
    assert torch.equal(again, loss) and torch.equal(saved, stats)
    assert all(torch.equal(x, y) for x, y in zip(backward(nb, c, stats), grads))


def test_training_stops(nb):
    """The command does not go on with gradients that are undefined."""
    from paper_2503_20591_b200 import train_policy
    nb.nbos_probe_towers_stall(SCORES, 2_000_000)
    with pytest.raises(RuntimeError, match="wait"):
        train_policy.train(hosts=64, snapshots=2, batch=50, steps=3, report=lambda text: None, table=False)
    nb.nbos_probe_towers_stall(-1, 0)
    assert nb.nbos_policy_towers_status() == nb.NBOS_OK


def test_taken_back(nb):
    import torch
    c = make(1, 30, 40, 16, 3, "float16", False, 8)
    want = forward(nb, c)
    nb.nbos_probe_towers_stall(SCORES, 1)
    nb.nbos_probe_towers_stall(-1, 1)
    assert all(torch.equal(x, y) for x, y in zip(forward(nb, c), want))
    for bad in (-2, 4):
        with pytest.raises(nb.NbosError):
            nb.nbos_probe_towers_stall(bad, 1)
