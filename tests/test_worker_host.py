"""Host-side checks of the worker's C ABI (no GPU needed)."""
import ctypes
import os

import pytest

from paper_2209_00159_amd import orloj as O
from paper_2209_00159_amd import worker as W


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(O.LIB_PATH):
        from paper_2209_00159_amd import build
        build.build()
    return O.load()


def test_null_handles_are_rejected_without_touching_the_gpu(lib):
    out = ctypes.c_void_p(123)
    assert lib.orloj_worker_create(ctypes.byref(out), None) == O.ORLOJ_E_INVALID and out.value is None
    assert lib.orloj_worker_create(None, None) == O.ORLOJ_E_INVALID
    assert lib.orloj_worker_sync(None) == O.ORLOJ_E_INVALID
    lib.orloj_worker_destroy(None)
    ad, c, b, v = O.AdapterSet(), O.PagedCache(), O.BatchRows(), O.Vectors()
    assert lib.orloj_worker_adapt(None, ad, 0, None, None, 0, None, 0, None, 0) == O.ORLOJ_E_INVALID
    assert lib.orloj_worker_cache_write(None, c, b, 0, v, v) == O.ORLOJ_E_INVALID
    assert lib.orloj_worker_cache_read(None, c, b, 0, v, v) == O.ORLOJ_E_INVALID
    assert lib.orloj_worker_attend(None, c, b, 1, 1, 1.0, v, None, v, None) == O.ORLOJ_E_INVALID


def test_padded_dimension():
    assert [W.dim_pad(d) for d in (1, 63, 64, 65, 128, 129, 256)] == [64, 64, 64, 128, 128, 192, 256]
