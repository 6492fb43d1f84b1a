"""Which kernel a product in 8 bits takes, and workspaces that have to be asked for: on the host, before the first HIP call (no GPU; the pointers passed are never dereferenced)."""
import ctypes as C
import os

import pytest

from test_more_operators_abi import EINVAL, ESMALL, FAKE, LIB, caller, i32, i64, sz, vp


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB):
        from paper_2403_07339_amd import build
        build.build()
    return C.CDLL(LIB)


@pytest.fixture(scope="module")
def cut(lib):
    tile, parts = i32(), i32()
    call = caller(lib.imunpack_diag_block8_cut, [i64, i64, i64, i32, vp, vp], dict(m=10, n=20, k=200, dtype=0, tile=C.addressof(tile), parts=C.addressof(parts)))

    def run(**change):
        code = call(**change)
        return (tile.value, parts.value) if code == 0 else code
    return run


def test_refusals(cut):
    for bad in (dict(m=-1), dict(n=-1), dict(k=0), dict(m=(1 << 24) + 1), dict(n=(1 << 24) + 1), dict(k=(1 << 24) + 1), dict(dtype=2), dict(tile=None), dict(parts=None)):
        assert cut(**bad) == EINVAL, bad


def test_a_product_that_is_cut_needs_its_workspace(lib, cut):
    size = sz()
    ws = caller(lib.imunpack_block8_gemm_workspace, [i64, i64, i64, i32, vp], dict(m=128, n=128, k=1 << 16, dtype=0, out=C.addressof(size)))
    call = caller(lib.imunpack_block8_gemm, [vp, i64, vp, i64, i32, vp, i64, vp, i64, i32, i64, i64, i64, vp, vp, i64, i32, vp, sz, vp],
                  dict(a=FAKE, lda=1 << 16, sa=FAKE, ldsa=512, fa=0, b=FAKE, ldb=1 << 16, sb=FAKE, ldsb=512, fb=0, m=128, n=128, k=1 << 16, bias=None, out=FAKE, ldo=128, dtype=0, ws=FAKE, bytes=1 << 30, st=None))
    for dtype in (0, 1):
        assert ws(dtype=dtype) == 0
        parts = cut(m=128, n=128, k=1 << 16, dtype=dtype)[1]
        assert parts > 1 and size.value == parts * 128 * 128 * 4
        assert call(dtype=dtype, bytes=size.value - 1) == ESMALL and call(dtype=dtype, ws=None) == EINVAL and call(dtype=dtype, ws=FAKE + 8) == EINVAL


def test_rows_of_logits_that_are_cut_need_their_workspace(lib):
    size = sz()
    ws = caller(lib.imunpack_logprobs_workspace, [i64, i64, i64, i64, i32, vp], dict(rows=2, vocab=128000, count=1, top=5, dtype=0, out=C.addressof(size)))
    call = caller(lib.imunpack_logprobs, [vp, i64, i64, i64, i32, vp, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, sz, vp],
                  dict(l=FAKE, ldl=128000, rows=2, vocab=128000, dtype=0, t=FAKE, count=1, ignore=-100, top=5, logp=FAKE, lse=FAKE, stats=FAKE, h=FAKE, tl=FAKE, ti=FAKE, ws=FAKE, bytes=1 << 30, st=None))
    for dtype in (0, 1):
        assert ws(dtype=dtype) == 0 and size.value > 0
        assert call(dtype=dtype, bytes=size.value - 1) == ESMALL and call(dtype=dtype, ws=None) == EINVAL and call(dtype=dtype, ws=FAKE + 4) == EINVAL


def test_few_rows_take_what_was_measured_as_the_faster(cut):
    """(rows, columns, places; fp32 or bfloat16): the kernel for few rows where a CU has one workgroup of it or one row to multiply, parts where it has several and sixteen rows."""
    for m, n, k, dtype in ((16, 4096, 4096, 0), (16, 4096, 4096, 1), (1, 11008, 4096, 0), (1, 8192, 4096, 0), (16, 2048, 4096, 1), (16, 1024, 1024, 0)):
        assert cut(m=m, n=n, k=k, dtype=dtype) == (0, 1), (m, n, k, dtype)
    for m, n, k, dtype in ((16, 11008, 4096, 0), (16, 11008, 4096, 1), (16, 8192, 4096, 0), (16, 8192, 4096, 1), (16, 11008, 11008, 0), (16, 5120, 4096, 0)):
        tile, parts = cut(m=m, n=n, k=k, dtype=dtype)
        assert tile == 1 and parts > 1, (m, n, k, dtype)
