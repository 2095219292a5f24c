"""Executor selection from two host threads with clusters of different sizes: a block's shared memory goes by the cluster's size,
and neither thread may be refused because of the other."""
from __future__ import annotations

import threading

import pytest

pytestmark = pytest.mark.gpu


def test_two_threads_with_different_clusters():
    import ctypes

    import torch
    from paper_2503_20591_b200 import binding as nb, build as lib_build
    lib_build.build()
    lib = nb.load_library()
    m = 1 << 19
    refused, outputs, start = [], {}, threading.Barrier(2)

    def work(hosts):
        state = [torch.full((hosts,), v, dtype=torch.int32, device="cuda") for v in (8, 0, 0, 640, 128_000, 1_048_576)]
        requests = torch.tensor([[1, 16, 1000, 1024]], dtype=torch.int32, device="cuda").repeat(m, 1)
        replicas = (torch.arange(3 * m, device="cuda", dtype=torch.int32) % hosts).view(m, 3)
        executor, can_run = (torch.full((m,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
        cluster = nb.nbos_cluster_state(hosts, 3, *[a.data_ptr() for a in state])
        args = (ctypes.byref(cluster), requests.data_ptr(), replicas.data_ptr(), m, executor.data_ptr(), can_run.data_ptr(), None)
        start.wait()
        for i in range(10000):
            status = lib.nbos_select_executors(*args)
            if status != nb.NBOS_OK:
                refused.append((hosts, status, nb.nbos_last_error_detail()[:100]))
        torch.cuda.synchronize()
        outputs[hosts] = bool(((executor >= 0) & (executor < hosts) & (can_run == 7)).all())

    threads = [threading.Thread(target=work, args=(h,)) for h in (500, 4000)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not refused, (len(refused), refused[:2])
    assert outputs == {500: True, 4000: True}
