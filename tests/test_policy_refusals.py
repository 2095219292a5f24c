"""What the policy entry points refuse. Arguments are checked before the device is looked at, so this runs without one;
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


def table(data=FAKE, rows=8, stride=64, n=64, dtype=nb.NBOS_F32):
    return nb.nbos_logits(data, rows, stride, n, dtype)


BAD_TABLES = [
    (table(data=0), "data is NULL"), (table(data=FAKE + 2), "aligned"), (table(data=FAKE + 1, dtype=nb.NBOS_BF16), "aligned"),
    (table(dtype=3), "dtype"), (table(dtype=-1), "dtype"), (table(n=0), "n_hosts"), (table(n=nb.NBOS_MAX_HOSTS + 1), "n_hosts"),
    (table(rows=-1), "rows"), (table(rows=1 << 31), "rows"), (table(stride=63), "row_stride"), (table(stride=-64), "row_stride"),
]


def distill(lib, t, hosts=FAKE, teacher=FAKE, tstride=3, k=3, T=1.0, grad_loss=None, loss=FAKE, stats=None, grad=None, gstride=64):
    return lib.nbos_policy_distill(ctypes.byref(t), hosts, teacher, tstride, k, T, grad_loss, 1.0, loss, stats, grad, gstride, None)


def balance(lib, t, groups=1, hosts=FAKE, k=3, loss=FAKE, counts=FAKE, shares=None, stats=None, grad=None, gstride=64):
    return lib.nbos_policy_balance(ctypes.byref(t), groups, hosts, k, None, 1.0, loss, counts, shares, stats, grad, gstride, None)


def sample(lib, t, u=FAKE, temperature=None, top_k=None, top_p=None, min_p=None, draws=3, hosts=FAKE, found=None):
    return lib.nbos_policy_sample(ctypes.byref(t), u, temperature, top_k, top_p, min_p, draws, hosts, found, None)


def refused(status, word):
    assert status == nb.NBOS_ERR_INVALID_ARG
    assert word in nb.nbos_last_error_detail(), nb.nbos_last_error_detail()


@pytest.mark.parametrize("t,word", BAD_TABLES)
def test_bad_tables(lib, t, word):
    refused(distill(lib, t), word)
    refused(balance(lib, t), word)
    refused(sample(lib, t), word)
    for call in (lambda: lib.nbos_policy_distill_backward(ctypes.byref(t), FAKE, FAKE, 3, 3, 1.0, FAKE, None, 1.0, FAKE, 64, None),
                 lambda: lib.nbos_policy_balance_backward(ctypes.byref(t), 1, FAKE, 3, FAKE, None, 1.0, FAKE, 64, None)):
        refused(call(), word)


def test_null_tables(lib):
    refused(lib.nbos_policy_distill(None, FAKE, FAKE, 3, 3, 1.0, None, 1.0, FAKE, None, None, 0, None), "logits is NULL")
    refused(lib.nbos_policy_balance(None, 1, FAKE, 3, None, 1.0, FAKE, FAKE, None, None, None, 0, None), "logits is NULL")
    refused(lib.nbos_policy_sample(None, FAKE, None, None, None, None, 1, FAKE, None, None), "logits is NULL")


@pytest.mark.parametrize("kw,word", [
    (dict(k=0), "k must"), (dict(k=nb.NBOS_POLICY_MAX_K + 1), "k must"), (dict(T=0.0), "temperature"),
    (dict(T=-1.0), "temperature"), (dict(T=float("nan")), "temperature"), (dict(T=float("inf")), "temperature"),
    (dict(T=1e-39), "temperature"), (dict(T=1e30), "temperature"), (dict(tstride=2), "teacher_stride"),
    (dict(tstride=-3), "teacher_stride"), (dict(hosts=None), "hosts is NULL"), (dict(hosts=FAKE + 2), "4-byte"),
    (dict(teacher=FAKE + 1), "4-byte"), (dict(grad_loss=FAKE + 2), "4-byte"), (dict(loss=FAKE + 2), "4-byte"),
    (dict(stats=FAKE + 2), "4-byte"), (dict(loss=None), "no output"), (dict(grad=FAKE * 2, gstride=63), "grad_stride"),
    (dict(grad=FAKE * 2 + 2), "aligned"), (dict(grad=FAKE, gstride=128), "row_stride"),
])
def test_bad_distill_arguments(lib, kw, word):
    refused(distill(lib, table(), **kw), word)


@pytest.mark.parametrize("kw,word", [
    (dict(k=0), "k must"), (dict(k=nb.NBOS_POLICY_MAX_K + 1), "k must"), (dict(groups=0), "n_groups"),
    (dict(groups=65536), "n_groups"), (dict(groups=3), "multiple"), (dict(hosts=None), "hosts is NULL"),
    (dict(loss=None), "NULL"), (dict(counts=None), "NULL"), (dict(counts=FAKE + 1), "4-byte"),
    (dict(shares=FAKE + 1), "4-byte"), (dict(stats=FAKE + 1), "4-byte"), (dict(grad=FAKE * 2, gstride=1), "grad_stride"),
    (dict(grad=FAKE, gstride=65), "row_stride"),
])
def test_bad_balance_arguments(lib, kw, word):
    refused(balance(lib, table(), **kw), word)


def test_balance_counts_fit_31_bits(lib):
    refused(balance(lib, table(rows=1 << 30), k=2), "31 bits")


@pytest.mark.parametrize("kw,word", [
    (dict(draws=0), "draws"), (dict(draws=nb.NBOS_POLICY_MAX_DRAWS + 1), "draws"), (dict(u=None), "NULL"),
    (dict(hosts=None), "NULL"), (dict(u=FAKE + 2), "4-byte"), (dict(temperature=FAKE + 2), "4-byte"),
    (dict(top_k=FAKE + 2), "4-byte"), (dict(top_p=FAKE + 2), "4-byte"), (dict(min_p=FAKE + 2), "4-byte"),
    (dict(found=FAKE + 2), "4-byte"),
])
def test_bad_sample_arguments(lib, kw, word):
    refused(sample(lib, table(), **kw), word)


def test_backward_needs_its_statistics(lib):
    t = table()
    refused(lib.nbos_policy_distill_backward(ctypes.byref(t), FAKE, FAKE, 3, 3, 1.0, None, None, 1.0, FAKE, 64, None), "stats")
    refused(lib.nbos_policy_distill_backward(ctypes.byref(t), FAKE, FAKE, 3, 3, 1.0, FAKE, None, 1.0, None, 64, None), "stats")
    refused(lib.nbos_policy_balance_backward(ctypes.byref(t), 1, FAKE, 3, None, None, 1.0, FAKE, 64, None), "stats")


def test_the_binding_refuses_wrong_tensors():
    """Types, devices and shapes are refused in Python, before any pointer is taken."""
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="cuda"):
        nb.nbos_policy_distill(x, torch.zeros(4, 3, dtype=torch.int32), None, torch.zeros(4))
    with pytest.raises(TypeError, match="float32"):
        nb.nbos_policy_sample(x.double(), torch.zeros(4, 1), torch.zeros(4, 1, dtype=torch.int32))
    with pytest.raises(TypeError, match="float32"):
        nb.nbos_policy_balance([1.0], None, None, None)
