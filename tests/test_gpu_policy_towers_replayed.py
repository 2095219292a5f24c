"""Steps that follow one another without a pause: captured many to a graph and replayed, each launch starts while the one before it ends. The pair of
blocks of a tile allocates tensor memory together, so both have to be there; a launch that went ahead waited for good once in some thousands."""
from __future__ import annotations

import pytest

from test_gpu_policy_towers import make, nb   # noqa: F401 (nb is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("groups,rows,hosts,width,k,mask,dtype", [(1, 2000, 3000, 64, 32, True, "bfloat16"), (1, 700, 300, 200, 3, False, "float16"), (3, 40, 5000, 64, 9, True, "float16"),
                                                                  (16, 64, 64, 32, 1, True, "bfloat16")])
def test_many_steps_in_a_row(nb, groups, rows, hosts, width, k, mask, dtype):
    import torch
    c = make(groups, rows, hosts, width, k, dtype, mask, 3)
    args, fit = (c["requests"], c["host_vectors"], c["hosts"], c["teacher_logits"]), dict(asks=c["asks"], room=c["room"])
    loss, stats = torch.empty(groups, rows, device="cuda"), torch.empty(groups, rows, 2 + k, device="cuda")
    grads = [torch.empty_like(t, memory_format=torch.contiguous_format) for t in args[:2]]

    def step(values):
        nb.nbos_policy_towers(*args, loss, stats, **fit)
        nb.nbos_policy_towers_backward(*args, stats, *grads, **fit, gradient_values=values)

    step(2)
    want = [t.clone() for t in (loss, stats, *grads)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for i in range(40):
            step(2 - i % 2)
        step(2)
    for t in (loss, stats, *grads):
        t.fill_(-7)
    for _ in range(40):
        graph.replay()
    assert nb.nbos_policy_towers_status() == nb.NBOS_OK
    assert all(torch.equal(x, y) for x, y in zip((loss, stats, *grads), want))


def test_two_streams_at_once(nb):
    """Calls on two streams whose launches take turns on the same multiprocessors: each gets what it gets alone."""
    import torch
    cases = [make(1, 1500, 2500, 64, 9, "bfloat16", True, 5), make(2, 300, 4000, 200, 3, "float16", False, 6)]
    streams = [torch.cuda.Stream() for _ in cases]

    def step(c):
        shape, k = c["hosts"].shape[:-1], c["hosts"].shape[-1]
        args, fit = (c["requests"], c["host_vectors"], c["hosts"], c["teacher_logits"]), dict(asks=c["asks"], room=c["room"])
        loss, stats = torch.empty(shape, device="cuda"), torch.empty((*shape, 2 + k), device="cuda")
        grads = [torch.empty_like(t, memory_format=torch.contiguous_format) for t in args[:2]]
        nb.nbos_policy_towers(*args, loss, stats, **fit)
        nb.nbos_policy_towers_backward(*args, stats, *grads, **fit)
        return loss, stats, *grads

    want = [step(c) for c in cases]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(60):
        for c, stream, results in zip(cases, streams, got):
            with torch.cuda.stream(stream):
                results.append(step(c))
    torch.cuda.synchronize()
    for results, ref in zip(got, want):
        assert all(torch.equal(x, y) for r in results for x, y in zip(r, ref))
    assert nb.nbos_policy_towers_status() == nb.NBOS_OK
