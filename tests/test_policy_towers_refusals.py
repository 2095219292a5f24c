"""What the two-tower entry points refuse. Arguments are checked before the device is looked at, so this runs without one;
no call here reaches a kernel."""
from __future__ import annotations

import ctypes

import pytest
import torch

from paper_2503_20591_b200 import binding as nb, build as lib_build

FAKE = 1 << 20   # an address that is aligned and never read


@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    return nb.load_library()


def towers(requests=FAKE, hosts=FAKE, rows=8, stride=64, gstride=512, hstride=64, hgstride=6400, groups=2, n=100, width=64,
           dtype=nb.NBOS_BF16, asks=None, room=None):
    return nb.nbos_towers(requests, hosts, rows, stride, gstride, hstride, hgstride, groups, n, width, dtype, asks, room)


def forward(lib, t, ids=FAKE, teacher=FAKE, tstride=3, k=3, T=1.0, loss=FAKE, stats=None):
    return lib.nbos_policy_towers(ctypes.byref(t), ids, teacher, tstride, k, T, loss, stats, None)


def backward(lib, t, ids=FAKE, teacher=FAKE, tstride=3, k=3, T=1.0, stats=FAKE, gl=None, ga=FAKE, gas=64, gag=512, gb=FAKE, gbs=64, gbg=6400):
    return lib.nbos_policy_towers_backward(ctypes.byref(t), ids, teacher, tstride, k, T, stats, gl, 1.0, ga, gas, gag, gb, gbs, gbg, None)


def refused(status, word):
    assert status == nb.NBOS_ERR_INVALID_ARG
    assert word in nb.nbos_last_error_detail(), nb.nbos_last_error_detail()


@pytest.mark.parametrize("kw,word", [
    (dict(dtype=nb.NBOS_F32), "BF16"), (dict(dtype=7), "BF16"), (dict(n=0), "n_hosts"), (dict(n=nb.NBOS_MAX_HOSTS + 1), "n_hosts"),
    (dict(width=0), "width"), (dict(width=nb.NBOS_POLICY_MAX_WIDTH + 1), "width"), (dict(groups=0), "n_groups"),
    (dict(groups=65536), "n_groups"), (dict(rows=-1), "rows"), (dict(rows=1 << 30), "rows"), (dict(stride=63), "request_stride"),
    (dict(hstride=63), "host_stride"), (dict(hstride=-64), "host_stride"), (dict(gstride=-1), "group strides"),
    (dict(hgstride=1 << 50), "group strides"), (dict(requests=None), "NULL"), (dict(hosts=None), "NULL"),
    (dict(requests=FAKE + 1), "aligned"), (dict(hosts=FAKE + 1), "aligned"), (dict(asks=FAKE), "together"), (dict(room=FAKE), "together"),
    (dict(asks=FAKE + 4, room=FAKE), "16-byte"), (dict(asks=FAKE, room=FAKE + 8), "16-byte"),
])
def test_bad_towers(lib, kw, word):
    refused(forward(lib, towers(**kw)), word)
    refused(backward(lib, towers(**kw)), word)


@pytest.mark.parametrize("kw,word", [
    (dict(k=0), "k must"), (dict(k=nb.NBOS_POLICY_MAX_K + 1), "k must"), (dict(T=0.0), "temperature"), (dict(T=float("nan")), "temperature"),
    (dict(T=float("inf")), "temperature"), (dict(T=1e-39), "temperature"), (dict(tstride=2), "teacher_stride"), (dict(ids=None), "hosts is NULL"),
    (dict(ids=FAKE + 2), "4-byte"), (dict(teacher=FAKE + 1), "4-byte"), (dict(stats=FAKE + 2), "4-byte"),
])
def test_bad_arguments(lib, kw, word):
    refused(forward(lib, towers(), **kw), word)
    refused(backward(lib, towers(), **kw), word)


def test_outputs(lib):
    refused(forward(lib, towers(), loss=None), "no output")
    refused(forward(lib, towers(), loss=FAKE + 2), "4-byte")
    refused(backward(lib, towers(), ga=None, gb=None), "no output")
    refused(backward(lib, towers(), stats=None), "stats")
    refused(backward(lib, towers(), gl=FAKE + 2), "4-byte")
    for kw, word in ((dict(ga=FAKE + 1), "aligned"), (dict(gas=63), "row stride"), (dict(gag=100), "overlap"), (dict(gbs=1), "row stride"),
                     (dict(gbg=0), "overlap"), (dict(gb=FAKE + 1), "aligned")):
        refused(backward(lib, towers(), **kw), word)
    refused(lib.nbos_policy_towers(None, FAKE, FAKE, 3, 3, 1.0, FAKE, None, None), "towers is NULL")
    assert forward(lib, towers(rows=0)) == nb.NBOS_OK


def test_the_binding_refuses_wrong_tensors():
    from paper_2503_20591_b200 import policy
    x, ids = torch.zeros(4, 8), torch.zeros(4, 3, dtype=torch.int32)
    with pytest.raises(TypeError, match="bfloat16"):
        nb.nbos_policy_towers(x, x, ids, None, torch.zeros(4))
    with pytest.raises(ValueError, match="cuda"):
        nb.nbos_policy_towers(x.bfloat16(), x.bfloat16(), ids, None, torch.zeros(4))
    with pytest.raises(ValueError, match="detach"):
        policy.tower_distill_loss(x.bfloat16(), x.bfloat16(), ids, torch.zeros(4, 3, requires_grad=True))
