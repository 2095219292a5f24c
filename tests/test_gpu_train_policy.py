"""What training feeds the operators with."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu


def test_the_balance_loss_sees_the_policys_own_answers(monkeypatch):
    """Training takes the load from hosts that were sampled from the logits it is about to change, not from the teacher's."""
    import torch
    from paper_2503_20591_b200 import build as lib_build, policy, train_policy
    lib_build.build()
    sampled, balanced = [], []
    sample, balance = policy.sample_hosts, policy.balance_loss

    def sample_hosts(logits, *args, **kw):
        out = sample(logits, *args, **kw)
        sampled.append((logits.data_ptr(), out[0].clone()))
        return out

    def balance_loss(logits, hosts):
        if logits.requires_grad:
            balanced.append((logits.data_ptr(), hosts.clone()))
        return balance(logits, hosts)

    monkeypatch.setattr(policy, "sample_hosts", sample_hosts)
    monkeypatch.setattr(policy, "balance_loss", balance_loss)
    train_policy.train(hosts=64, snapshots=3, batch=100, steps=4, report=lambda text: None)
    assert len(balanced) == 4 and len(sampled) == 5
    for (x, hosts), (y, drawn) in zip(balanced, sampled):
        assert x == y and torch.equal(hosts, drawn)
