"""Arguments of siso_kv.h that are refused before any call into the GPU's runtime."""

import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def siso():
    if not os.path.exists(os.path.join(ROOT, "paper_2508_18736_amd", "libsiso.so")):
        from paper_2508_18736_amd import build
        build.build(verbose=False)
    from paper_2508_18736_amd import siso as m
    return m


@pytest.mark.parametrize("layers,kv_heads,head_dim,page_tokens,pages,dtype", [
    (0, 2, 64, 16, 4, 1), (1, 0, 64, 16, 4, 1), (1, 2, 12, 16, 4, 1), (1, 2, 264, 16, 4, 1), (1, 2, 64, 8, 4, 1), (1, 2, 64, 48, 4, 1),
    (1, 2, 64, 2048, 4, 1), (1, 2, 64, 16, 0, 1), (1, 2, 64, 16, 4, 0), (1, 1025, 64, 16, 4, 1), (1, 2, 64, 16, 4, 7)])
def test_caches_that_are_not_made(siso, layers, kv_heads, head_dim, page_tokens, pages, dtype):
    assert (siso.F32, siso.BF16) == (0, 1)
    h = C.c_void_p()
    assert siso._lib.siso_kv_create(layers, kv_heads, head_dim, page_tokens, pages, dtype, C.byref(h)) == siso.EINVAL
    assert not h.value


def test_no_handle(siso):
    lib = siso._lib
    assert lib.siso_kv_create(1, 2, 64, 16, 4, siso.BF16, None) == siso.EINVAL
    batch = siso._KvBatchStruct(1, 1, None, None, None, 0, 0, 0)
    assert lib.siso_kv_set_stream(None, None) == siso.EINVAL
    assert lib.siso_kv_write(None, 0, C.byref(batch), None, 0, 0, None, 0, 0) == siso.EINVAL
    assert lib.siso_kv_read(None, 0, C.byref(batch), siso.BF16, None, None) == siso.EINVAL
    assert lib.siso_kv_attend(None, 0, C.byref(batch), None, 0, 0, 2, 1.0, 0, None, None) == siso.EINVAL
    assert lib.siso_kv_verify(None, C.byref(batch), None, 10, siso.F32, None, 0, None, 0, None, None, None, None) == siso.EINVAL
    assert lib.siso_kv_bad_pages(None) == siso.EINVAL
    lib.siso_kv_destroy(None)
