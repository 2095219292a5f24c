"""Executor selection's first call in a process, on memory that is new to it: stages of the ring are not given back before they have
been read. Each process compares its first call with its third on the same inputs, and the first results with the oracle's."""
from __future__ import annotations

import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = """
import numpy as np, torch
import oracle
from paper_2503_20591_b200 import binding as nb
rng = np.random.default_rng({seed})
hosts, m = {hosts}, {m}
gpus = rng.integers(1, 9, hosts)
state = [gpus, gpus * rng.integers(0, 4, hosts), rng.integers(0, gpus + 1), 16 * gpus, rng.choice([4000, 16000, 64000], hosts), rng.choice([2048, 65536, 1 << 20], hosts)]
state = [np.ascontiguousarray(a, dtype=np.int32) for a in state]
g = rng.integers(0, 9, m)
req = np.stack([g, 16 * g, rng.choice([1000, 4000, 16000], m), rng.choice([1024, 65536], m)], axis=1).astype(np.int32)
rep = rng.integers(0, hosts, (m, 3)).astype(np.int32)
dev = [torch.from_numpy(a).cuda() for a in state]
r, p = torch.from_numpy(req).cuda(), torch.from_numpy(rep).cuda()
outs = [[torch.full((m,), -9, dtype=torch.int32, device="cuda") for _ in range(2)] for _ in range(3)]
for ex, mask in outs:
    nb.nbos_select_executors(*dev, r, p, ex, mask)
torch.cuda.synchronize()
n = 200_000
ref = oracle.select_executors(*state, req[:n], rep[:n])
for ex, mask in outs:
    assert torch.equal(ex, outs[2][0]) and torch.equal(mask, outs[2][1]), int((mask != outs[2][1]).sum())
    assert np.array_equal(ex[:n].cpu().numpy(), ref[0]) and np.array_equal(mask[:n].cpu().numpy(), ref[1])
"""


def test_the_first_call_is_right():
    from paper_2503_20591_b200 import build as lib_build
    lib_build.build()
    for seed in range(6):
        done = subprocess.run([sys.executable, "-c", CODE.format(seed=seed, hosts=4096, m=2_500_000)], cwd=ROOT, capture_output=True, text=True, timeout=120)
        assert done.returncode == 0, done.stderr[-2000:]
