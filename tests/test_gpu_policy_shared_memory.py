"""Calls whose blocks take just under 48 KB of dynamic shared memory, the limit that a kernel has unless it asks for more. That limit
holds for the static part too, and what a kernel has asked for stays with it for the life of the process: so each list of
calls below runs in a process of its own, one call per instance of a kernel, and their answers are compared with the 64-bit oracle
within the tolerances derived in test_gpu_policy.py."""
from __future__ import annotations

import os
import subprocess
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# (hosts, type, call); 300 rows: two for each SM, as the block forms want
DISTILL = [(4000, "float32", "fused"), (8000, "bfloat16", "fused"), (8000, "float16", "fused"),
           (4072, "float32", "backward"), (8144, "bfloat16", "backward"), (8144, "float16", "backward")]
BALANCE = [(4000, "float32", "fused"), (6000, "bfloat16", "fused"), (6000, "float16", "fused"),
           (3900, "float32", "backward"), (5800, "bfloat16", "backward"), (5800, "float16", "backward")]
SMALL = [(360, "float32", "fused"), (361, "bfloat16", "fused"), (360, "float16", "fused"),
         (361, "float32", "backward"), (360, "bfloat16", "backward"), (361, "float16", "backward")]
LISTS = {"distill": DISTILL, "balance": BALANCE, "small": SMALL}


def calls(which):
    sys.path[:0] = [ROOT, os.path.join(ROOT, "tests")]
    import test_gpu_policy as base
    from paper_2503_20591_b200 import binding as nb
    failures = 0
    for n, dtype, call in LISTS[which]:
        rng = np.random.default_rng(n)
        rows, k = (100 if which == "small" else 300), 3
        x, x64 = base.make_logits(rng, rows, n, dtype)
        hosts = base.make_hosts(rng, rows, n, k)
        try:
            if which == "distill":
                teacher, gl = rng.normal(size=(rows, k)).astype(np.float32), np.ones(rows, np.float32)
                loss, grad, tol_l, tol_g = base.distill_bounds(x64, hosts, teacher.astype(np.float64), 1.5, np.ones(rows), dtype)
                got = base.run_distill(nb, x, hosts, teacher, 1.5, 1.0, gl, backward=call == "backward")
                base.close(got[0], loss, tol_l)
                base.close(got[1], grad, tol_g)
            else:
                base.check_balance(nb, x[None], x64[None], hosts[None], 64.0, np.ones(1, np.float32), dtype, backward=call == "backward")
        except (nb.NbosError, AssertionError) as e:
            failures += 1
            print(f"{which} {call} {rows} x {n} {dtype}: {str(e)[:200]}")
    return failures


@pytest.mark.gpu
@pytest.mark.parametrize("which", sorted(LISTS))
def test_first_calls_of_a_process_near_the_limit(which):
    done = subprocess.run([sys.executable, os.path.abspath(__file__), which], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert done.returncode == 0, done.stdout + done.stderr[-2000:]


@pytest.mark.gpu
def test_two_threads_with_different_sizes():
    """Two host threads in the same kernel, one with 54 KB a block and one with 96 KB: neither may be refused because of the other."""
    import threading

    import torch
    from paper_2503_20591_b200 import binding as nb, build as lib_build
    lib_build.build()
    nb.load_library()
    refused, start = [], threading.Barrier(2)

    def work(n):
        x = torch.zeros((300, n), dtype=torch.bfloat16, device="cuda")
        hosts = torch.zeros((300, 3), dtype=torch.int32, device="cuda")
        loss, grad = torch.empty(300, device="cuda"), torch.empty_like(x)
        even, counts = torch.empty(1, device="cuda"), torch.empty((1, n), dtype=torch.int32, device="cuda")
        start.wait()
        for _ in range(1500):
            try:
                nb.nbos_policy_distill(x, hosts, None, loss, out_grad=grad)
                nb.nbos_policy_balance(x, hosts, even, counts, out_grad=grad)
            except nb.NbosError as e:
                refused.append((n, str(e)[:100]))
        torch.cuda.synchronize()

    threads = [threading.Thread(target=work, args=(n,)) for n in (9000, 16000)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not refused, (len(refused), refused[:2])


if __name__ == "__main__":
    sys.exit(min(1, calls(sys.argv[1])))
