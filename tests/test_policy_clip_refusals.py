"""What nbos_policy_clip refuses, before the device is looked at; no call here reaches a kernel."""
from __future__ import annotations

import ctypes

import pytest

from paper_2503_20591_b200 import binding as nb, build as lib_build

FAKE = 1 << 20   # an address that is aligned and never read


@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    return nb.load_library()


def call(lib, data=(FAKE, FAKE), out=(FAKE, FAKE), numel=(8, 8), dtype=(nb.NBOS_F32, nb.NBOS_BF16), n=None, max_norm=1.0, kind=nb.NBOS_NORM_2,
         norm=FAKE):
    arr = lambda t, v: None if v is None else ctypes.addressof(keep.setdefault(t, (t * len(v))(*v))) if t is not ctypes.c_void_p else \
        ctypes.addressof(hold.append((t * len(v))(*v)) or hold[-1])
    keep, hold = {}, []
    return lib.nbos_policy_clip(arr(ctypes.c_void_p, data), arr(ctypes.c_void_p, out), arr(ctypes.c_int64, numel), arr(ctypes.c_int32, dtype),
                                len(data or ()) if n is None else n, max_norm, kind, norm, None)


@pytest.mark.parametrize("kw,word", [
    (dict(n=-1), "n_tensors"), (dict(data=None, n=2), "NULL"), (dict(numel=None), "NULL"), (dict(dtype=None), "NULL"), (dict(kind=2), "norm_kind"),
    (dict(max_norm=-1.0), "max_norm"), (dict(max_norm=float("nan")), "max_norm"), (dict(out=None, norm=None), "no output"),
    (dict(norm=FAKE + 2), "4-byte"), (dict(dtype=(0, 3)), "tensor 1: unknown dtype"), (dict(numel=(8, -1)), "tensor 1: numel"),
    (dict(numel=(1 << 41, 8)), "tensor 0: numel"), (dict(data=(FAKE, None)), "tensor 1 is NULL"), (dict(out=(None, FAKE)), "tensor 0 is NULL"),
    (dict(data=(FAKE + 2, FAKE)), "tensor 0 is not aligned"), (dict(out=(FAKE, FAKE + 1)), "tensor 1 is not aligned"),
])
def test_bad_arguments(lib, kw, word):
    assert call(lib, **kw) == nb.NBOS_ERR_INVALID_ARG
    assert word in nb.nbos_last_error_detail(), nb.nbos_last_error_detail()
