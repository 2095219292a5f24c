"""The balance loss of tables with many rows and few hosts, or many chosen hosts a row: every SM takes part, whatever rows * hosts is."""
from __future__ import annotations

import numpy as np
import pytest

from test_gpu_policy import check_balance, make_hosts, make_logits, nb  # noqa: F401 (nb is a fixture)

pytestmark = pytest.mark.gpu


def test_narrow_tables_are_not_left_to_one_block(nb):  # noqa: F811
    """16.8 million chosen hosts of 65,536 rows: 10 ms by one block, 0.1 ms by all; anything below 2 ms will do."""
    import torch
    x = torch.zeros((65536, 1), device="cuda")
    hosts = torch.zeros((65536, 256), dtype=torch.int32, device="cuda")
    loss, counts = torch.empty(1, device="cuda"), torch.empty((1, 1), dtype=torch.int32, device="cuda")
    times = []
    for _ in range(5):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        nb.nbos_policy_balance(x, hosts, loss, counts)
        end.record()
        end.synchronize()
        times.append(begin.elapsed_time(end))
    assert int(counts) == 65536 * 256 and float(loss) == 1.0
    assert min(times) < 2.0, times


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,n", [(1024, 32), (1025, 32), (512, 64), (513, 64), (512, 33), (256, 256), (257, 256), (256, 65), (128, 512),
                                    (129, 512), (128, 257), (5000, 1), (3000, 2)])
def test_both_sides_of_the_border_between_the_forms(nb, rows, n, dtype):  # noqa: F811
    rng = np.random.default_rng(rows + n)
    x, x64 = make_logits(rng, rows, n, dtype)
    hosts = make_hosts(rng, rows, n, 3)[None]
    check_balance(nb, x[None], x64[None], hosts, 512.0 * rows / n, rng.normal(size=1).astype(np.float32), dtype)
    check_balance(nb, x[None], x64[None], hosts, 512.0 * rows / n, rng.normal(size=1).astype(np.float32), dtype, backward=True)
