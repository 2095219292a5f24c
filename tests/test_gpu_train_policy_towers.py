"""The training step without the table of scores, with residual blocks and clipping: it runs through the three operators, and its
gradients are those of the step with the table."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tp():
    from paper_2503_20591_b200 import build as lib_build, train_policy
    lib_build.build()
    return train_policy


def test_room_is_the_rules_own_test(tp):
    """asks <= room, four by four, says what Cluster.fits says."""
    import torch
    from paper_2503_20591_b200 import workloads
    for w in (workloads.what_if_sweep(6, 200, 300), workloads.mixed_gpu_cluster(333, 500, seed=3)):
        cluster = tp.Cluster(w)
        try:
            asks = torch.from_numpy(w.requests).cuda()
            inside = (asks[:, :, None] <= cluster.room[:, None]).all(-1) & (asks >= 0).all(-1)[..., None]
            assert torch.equal(inside, cluster.fits(asks))
        finally:
            cluster.close()


def test_gradients_with_and_without_the_table(tp):
    """Both losses on the same vectors. Vectors are 16-bit in both; the table's gradient goes back through 32-bit products, the
    other's G is rounded to bfloat16 (2^-8 relative an entry) and its result once more: 3 * 2^-8 of the sum of magnitudes."""
    import torch
    from paper_2503_20591_b200 import policy, workloads
    torch.manual_seed(1)
    w = workloads.what_if_sweep(4, 150, 200)
    cluster = tp.Cluster(w)
    try:
        requests = torch.from_numpy(w.requests).cuda()
        wanted = cluster.teacher(requests)
        teacher = torch.tensor(tp.TEACHER_LOGITS, device="cuda")
        net = tp.TwoTowerPolicy(4, cluster.features.shape[-1], blocks=2).cuda()
        a, b = (v.detach().bfloat16().requires_grad_(True) for v in net.vectors(tp.request_features(requests), cluster.features))
        loss = policy.tower_distill_loss(a, b, wanted, teacher, asks=requests, room=cluster.room)
        loss.sum().backward()
        x, y = a.detach().float().requires_grad_(True), b.detach().float().requires_grad_(True)
        logits = (x.double() @ y.double().transpose(1, 2)).float().masked_fill(~cluster.fits(requests), float("-inf"))
        logits.retain_grad()
        want = policy.distill_loss(logits, wanted, teacher)
        want.sum().backward()
        # 32-bit sums and powers of both: 2^-12 of a loss and its parts, which stay below 2^5
        torch.testing.assert_close(loss.detach(), want.detach(), rtol=0, atol=2.0 ** -7)
        g = logits.grad.abs()
        for got, ref, size in ((a.grad, x.grad, g @ y.detach().abs()), (b.grad, y.grad, g.transpose(1, 2) @ x.detach().abs())):
            assert ((got.float() - ref).abs() <= 3 * 2.0 ** -8 * size + 1e-6).all()
    finally:
        cluster.close()


@pytest.mark.parametrize("table,blocks,max_norm", [(False, 0, None), (False, 2, 0.5), (True, 1, 0.5)])
def test_training_runs(tp, monkeypatch, table, blocks, max_norm):
    import torch
    from paper_2503_20591_b200 import policy
    calls, norms = {"tower_distill_loss": 0, "block_norm": 0, "clip_gradients": 0}, []
    for name in calls:
        def counted(*args, _f=getattr(policy, name), _name=name, **kw):
            calls[_name] += 1
            out = _f(*args, **kw)
            if _name == "clip_gradients":
                grads = [p.grad for p in args[0] if p.grad is not None] if isinstance(args[0], list) else None
                norms.append((out, grads))
            return out
        monkeypatch.setattr(policy, name, counted)
    out = tp.train(hosts=64, snapshots=3, batch=100, steps=5, report=lambda text: None, blocks=blocks, max_norm=max_norm, table=table)
    assert calls["tower_distill_loss"] == (0 if table else 5)
    assert (calls["block_norm"] > 0) == (blocks > 0)
    assert calls["clip_gradients"] == (5 if max_norm else 0)
    assert all(torch.isfinite(n) and float(n) > 0 for n, _ in norms)
    assert out["feasible"] and out["distinct"]


def test_a_step_of_all_three_in_one_graph(tp):
    """Blocks, the loss without the table, their gradients and clipping, captured once and replayed on other requests."""
    import torch
    from paper_2503_20591_b200 import policy, workloads
    torch.manual_seed(2)
    w = workloads.what_if_sweep(3, 120, 90)
    cluster = tp.Cluster(w)
    try:
        net = tp.TwoTowerPolicy(4, cluster.features.shape[-1], blocks=1).cuda()
        teacher = torch.tensor(tp.TEACHER_LOGITS, device="cuda")
        first = torch.from_numpy(w.requests).cuda()
        second = first.flip(1).contiguous()
        requests, wanted = first.clone(), cluster.teacher(first)

        def step():
            net.zero_grad(set_to_none=True)
            a, b = (v.bfloat16() for v in net.vectors(tp.request_features(requests), cluster.features))
            policy.tower_distill_loss(a, b, wanted, teacher, asks=requests, room=cluster.room).mean().backward()
            return policy.clip_gradients(net.parameters(), 0.01)

        def eager(batch):
            requests.copy_(batch), wanted.copy_(cluster.teacher(batch))
            norm = step()
            return [norm.clone()] + [p.grad.clone() for p in net.parameters()]

        want = [eager(first), eager(second)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        scale = torch.tensor([8.0, 128.0, 16_000.0, 65_536.0], device="cuda")
        monkey, tp.request_features = tp.request_features, lambda r: r.float() / scale   # (no copy from the host while capturing)
        try:
            with torch.cuda.graph(graph):
                norm = step()
        finally:
            tp.request_features = monkey
        grads = [p.grad for p in net.parameters()]
        for batch, ref in ((second, want[1]), (first, want[0])):
            requests.copy_(batch), wanted.copy_(cluster.teacher(batch))
            graph.replay()
            torch.cuda.synchronize()
            for got, r in zip([norm] + grads, ref):
                torch.testing.assert_close(got, r, rtol=1e-5, atol=1e-7)   # torch's own products may sum in another order
    finally:
        cluster.close()
