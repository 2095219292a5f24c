"""Training without the table of scores holds no table of scores, in no step and not at the end either."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tp():
    from paper_2503_20591_b200 import build as lib_build, train_policy
    lib_build.build()
    return train_policy


def test_memory_stays_below_the_table(tp):
    """Two steps with a table of 2 x 8,192 x 16,384 scores: 1,074 MB in 32 bits, 268 MB as truth values. What PyTorch holds (vectors of 64
    and what gradients of them need: below 30 MB; 4 million scores at a time with their tests: below 200 MB) stays under the latter."""
    import torch
    torch.cuda.empty_cache()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    out = tp.train(hosts=16384, snapshots=2, batch=8192, steps=2, report=lambda text: None, table=False)
    assert torch.cuda.max_memory_allocated() - before < 2 * 8192 * 16384
    assert out["feasible"] and out["distinct"] and len(out["history"]) == 2


@pytest.mark.parametrize("table", [False, True])
def test_pieces_say_what_the_whole_says(tp, monkeypatch, table):
    """Pieces of snapshots and of requests, with shorter ones at the end. The library's product may sum in another order then, so a
    sample may differ: answers within 2 %."""
    results = []
    for piece in (1 << 22, 96 * 50, 96 * 7 * 3):   # all of it; 50 snapshots' worth of one request; 3 snapshots x 7 requests
        monkeypatch.setattr(tp, "PIECE", piece)
        results.append(tp.train(hosts=96, snapshots=5, batch=101, steps=3, report=lambda text: None, table=table))
    whole = results[0]
    for r in results[1:]:
        assert r["feasible"] and r["distinct"] and r["hosts_used_by_rule"] == whole["hosts_used_by_rule"]
        for k in ("agreement", "found", "hosts_used"):
            assert abs(r[k] - whole[k]) <= 0.02 * abs(whole[k]) + 0.02, k
        for x, y in zip(r["history"], whole["history"]):
            assert all(abs(a - b) <= 0.02 * abs(b) + 0.02 for a, b in zip(x, y))


def test_balance_is_the_losss_own(tp, monkeypatch):
    """What is put together from pieces is what the balance loss says of the whole table."""
    import torch
    from paper_2503_20591_b200 import policy
    calls, balance = [], policy.balance_loss

    def watched(logits, hosts):
        calls.append((logits.detach().clone(), hosts.clone()))
        return balance(logits, hosts)

    monkeypatch.setattr(policy, "balance_loss", watched)
    monkeypatch.setattr(tp, "PIECE", 96 * 5 * 30)   # 5 snapshots x 30 requests
    out = tp.train(hosts=96, snapshots=5, batch=100, steps=1, report=lambda text: None, table=False)
    pieces = calls[:8:2]                            # a call for the policy's hosts, one for the rule's, four pieces
    logits, hosts = (torch.cat(v, 1) for v in zip(*pieces))
    assert logits.shape == (5, 100, 96)
    # sums of 100 shares and 96 products in 32 bits on one side: below 1e-5 of the result
    assert abs(out["history"][0][1] - float(balance(logits, hosts)[0].mean())) <= 1e-4
