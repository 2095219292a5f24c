"""What nbos_policy_block_norm and its backward refuse, before the device is looked at; no call here reaches a kernel."""
from __future__ import annotations

import ctypes

import pytest

from paper_2503_20591_b200 import binding as nb, build as lib_build

FAKE = 1 << 20   # an address that is aligned and never read


@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    return nb.load_library()


def block(residual=FAKE, branch=FAKE, gate=FAKE, post=FAKE, pre=FAKE, rs=64, bs=64, gs=64, rows=8, per=4, width=64, dtype=nb.NBOS_BF16,
          gate_dtype=nb.NBOS_BF16, weight_dtype=nb.NBOS_F32, alpha=1.0, eps=1e-6):
    return nb.nbos_block(residual, branch, gate, post, pre, rs, bs, gs, rows, per, width, dtype, gate_dtype, weight_dtype, alpha, eps)


def forward(lib, b, out=FAKE, os=64, normed=FAKE, ns=64, stats=FAKE):
    return lib.nbos_policy_block_norm(ctypes.byref(b), out, os, normed, ns, stats, None)


def backward(lib, b, stats=FAKE, dr=FAKE, drs=64, dh=FAKE, dhs=64, gx=FAKE, gxs=64, gy=FAKE, gys=64, gg=FAKE, ggs=64, gpost=FAKE, gpre=FAKE):
    return lib.nbos_policy_block_norm_backward(ctypes.byref(b), stats, dr, drs, dh, dhs, gx, gxs, gy, gys, gg, ggs, gpost, gpre, None)


def refused(status, word):
    assert status == nb.NBOS_ERR_INVALID_ARG
    assert word in nb.nbos_last_error_detail(), nb.nbos_last_error_detail()


@pytest.mark.parametrize("kw,word", [
    (dict(dtype=5), "dtype"), (dict(gate_dtype=nb.NBOS_F16), "gate_dtype"), (dict(weight_dtype=nb.NBOS_F16), "weight_dtype"),
    (dict(width=0), "width"), (dict(width=nb.NBOS_BLOCK_MAX_WIDTH + 1), "width"), (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"),
    (dict(alpha=float("inf")), "residual_scale"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(residual=None), "residual is NULL"),
    (dict(branch=None), "branch is NULL"), (dict(residual=FAKE + 1), "aligned"), (dict(branch=FAKE + 1), "aligned"), (dict(rs=63), "residual"),
    (dict(bs=63), "branch"), (dict(per=0), "rows_per_gate"), (dict(per=3), "rows_per_gate"), (dict(gs=63), "gate"), (dict(gate=FAKE + 1), "gate"),
    (dict(post=FAKE + 2), "post_weight"), (dict(pre=FAKE + 1), "pre_weight"),
])
def test_bad_blocks(lib, kw, word):
    refused(forward(lib, block(**kw)), word)
    refused(backward(lib, block(**kw)), word)


def test_bad_arguments(lib):
    for kw, word in ((dict(out=FAKE + 1), "aligned"), (dict(os=63), "out_residual"), (dict(ns=1), "out_normed"), (dict(stats=FAKE + 2), "4-byte"),
                     (dict(out=None, normed=None, stats=None), "no output")):
        refused(forward(lib, block(), **kw), word)
    for kw, word in ((dict(stats=None), "stats"), (dict(stats=FAKE + 1), "4-byte"), (dict(dr=None, dh=None), "both NULL"), (dict(drs=63), "grad_residual"),
                     (dict(dhs=63), "grad_normed"), (dict(gxs=63), "out_grad_residual"), (dict(gys=63), "out_grad_branch"), (dict(ggs=63), "out_grad_gate"),
                     (dict(gx=FAKE + 1), "aligned"), (dict(gpost=FAKE + 2), "aligned"),
                     (dict(gx=None, gy=None, gg=None, gpost=None, gpre=None), "no output")):
        refused(backward(lib, block(), **kw), word)
    refused(backward(lib, block(gate=None)), "without a gate")
    refused(backward(lib, block(post=None)), "weight that is NULL")
    refused(backward(lib, block(pre=None)), "weight that is NULL")
    refused(lib.nbos_policy_block_norm(None, FAKE, 64, FAKE, 64, FAKE, None), "block is NULL")
    assert forward(lib, block(rows=0)) == nb.NBOS_OK
