"""The calls on tensors in 8-bit floating point and on rows of logits reject bad arguments on the host, before the first HIP call (no GPU; the pointers passed are
never dereferenced)."""
import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2403_07339_amd", "libimunpack.so")
EINVAL, ESMALL = -1, -5
vp, i64, i32, sz = C.c_void_p, C.c_int64, C.c_int, C.c_size_t
FAKE = 0x1000


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB):
        from paper_2403_07339_amd import build
        build.build()
    return C.CDLL(LIB)


def caller(f, types, good):
    f.restype, f.argtypes = C.c_int, types
    names = list(good)
    return lambda **change: f(*[{**good, **change}[k] for k in names])


def test_quantize(lib):
    call = caller(lib.imunpack_block8_quantize, [vp, i64, i64, i64, i32, i32, i32, vp, i64, vp, i64, vp, i64, vp, i64, vp],
                  dict(x=FAKE, ldx=200, rows=300, cols=200, dtype=0, fmt=0, square=0, q=FAKE, ldq=256, s=FAKE, lds=16, t=FAKE, ldt=384, ts=FAKE, ldts=16, st=None))
    for bad in (dict(x=None), dict(ldx=199), dict(rows=-1), dict(rows=(1 << 31) + 1), dict(rows=(1 << 24) + 1), dict(cols=0), dict(cols=(1 << 24) + 1), dict(dtype=2), dict(fmt=2), dict(fmt=-1),
                dict(q=None, t=None), dict(q=FAKE + 8), dict(s=None), dict(s=FAKE + 4), dict(ldq=200), dict(ldq=255), dict(ldq=264), dict(lds=1), dict(lds=17), dict(t=FAKE + 1), dict(ldt=256),
                dict(ts=None), dict(ldts=2), dict(ldts=24)):
        assert call(**bad) == EINVAL, bad
    assert call(rows=0, x=None, q=None, t=None) == 0


def test_turn_and_values(lib):
    call = caller(lib.imunpack_block8_turn, [vp, i64, vp, i64, i64, i64, i32, vp, i64, vp, i64, vp],
                  dict(q=FAKE, ldq=256, s=FAKE, lds=16, rows=300, cols=200, fmt=0, t=FAKE, ldt=384, ts=FAKE, ldts=16, st=None))
    for bad in (dict(q=None), dict(q=FAKE + 4), dict(s=None), dict(ldq=128), dict(lds=0), dict(rows=-1), dict(rows=(1 << 24) + 1), dict(cols=0), dict(fmt=3), dict(t=None), dict(ldt=300), dict(ts=None)):
        assert call(**bad) == EINVAL, bad
    assert call(rows=0) == 0
    call = caller(lib.imunpack_block8_values, [vp, i64, vp, i64, i64, i64, i32, vp, i64, i32, vp],
                  dict(q=FAKE, ldq=256, s=FAKE, lds=16, rows=3, cols=200, fmt=0, out=FAKE, ldo=200, dtype=0, st=None))
    for bad in (dict(q=None), dict(s=None), dict(ldq=192), dict(out=None), dict(ldo=199), dict(dtype=-1), dict(fmt=2), dict(rows=-2)):
        assert call(**bad) == EINVAL, bad
    assert call(rows=0, out=None) == 0


def test_gemm(lib):
    size = sz()
    ws = caller(lib.imunpack_block8_gemm_workspace, [i64, i64, i64, i32, vp], dict(m=10, n=20, k=200, dtype=0, out=C.addressof(size)))
    for bad in (dict(m=-1), dict(n=-1), dict(k=0), dict(m=(1 << 24) + 1), dict(n=(1 << 24) + 1), dict(k=(1 << 24) + 1), dict(dtype=2), dict(out=None)):
        assert ws(**bad) == EINVAL, bad
    assert ws() == 0
    call = caller(lib.imunpack_block8_gemm, [vp, i64, vp, i64, i32, vp, i64, vp, i64, i32, i64, i64, i64, vp, vp, i64, i32, vp, sz, vp],
                  dict(a=FAKE, lda=256, sa=FAKE, ldsa=16, fa=0, b=FAKE, ldb=256, sb=FAKE, ldsb=16, fb=0, m=10, n=20, k=200, bias=None, out=FAKE, ldo=20, dtype=0, ws=FAKE, bytes=1 << 30, st=None))
    for bad in (dict(a=None), dict(sa=None), dict(a=FAKE + 8), dict(lda=(1 << 24) + 16), dict(ldsa=(1 << 24) + 16), dict(lda=128), dict(lda=260), dict(ldsa=0), dict(ldsa=8), dict(fa=2), dict(b=None), dict(sb=None), dict(ldb=240), dict(ldsb=1),
                dict(fb=-1), dict(out=None), dict(ldo=19), dict(m=-1), dict(k=0), dict(dtype=3)):
        assert call(**bad) == EINVAL, bad
    assert call(m=0, a=None) == 0 and call(n=0, out=None) == 0
    # a product with few rows of a long contraction: if it takes a workspace, a smaller one is refused
    assert ws(m=128, n=128, k=1 << 16) == 0
    if size.value:
        big = dict(m=128, n=128, k=1 << 16, lda=1 << 16, ldb=1 << 16, ldsa=512, ldsb=512, ldo=128)
        assert call(**big, bytes=size.value - 1) == ESMALL and call(**big, ws=None) == EINVAL and call(**big, ws=FAKE + 8) == EINVAL


def test_act8(lib):
    call = caller(lib.imunpack_act8, [vp, i64, i64, i64, i32, i32, i32, vp, i64, vp, i64, vp, i64, vp, vp, i64, vp, vp, i64, vp],
                  dict(u=FAKE, ldu=400, rows=3, cols=200, dtype=0, act=0, gated=1, y=FAKE, ldy=200, q=FAKE, ldq=256, qs=FAKE, ldqs=16, k=FAKE, k2=FAKE, ldk=256, ks=FAKE, k2s=FAKE, ldks=16, st=None))
    for bad in (dict(u=None), dict(ldu=399), dict(rows=-1), dict(cols=0), dict(dtype=2), dict(act=2), dict(ldy=199), dict(y=None, q=None), dict(q=FAKE + 8), dict(ldq=208), dict(qs=None), dict(k=FAKE + 2),
                dict(k2=None), dict(ks=None), dict(k2s=None), dict(ldk=200), dict(ldks=1)):
        assert call(**bad) == EINVAL, bad
    assert call(rows=0, u=None) == 0
    call = caller(lib.imunpack_act8_backward, [vp, i64, i64, i64, i32, i32, i32, vp, vp, i64, vp, vp, i64, vp, i64, vp],
                  dict(g=FAKE, ldg=200, rows=3, cols=200, dtype=0, act=1, gated=1, k=FAKE, k2=FAKE, ldk=256, ks=FAKE, k2s=FAKE, ldks=16, gu=FAKE, ldgu=400, st=None))
    for bad in (dict(g=None), dict(ldg=100), dict(gu=None), dict(ldgu=399), dict(k=None), dict(k2=None), dict(ks=None), dict(k2s=None), dict(ldk=128), dict(act=-1), dict(dtype=7), dict(cols=-1)):
        assert call(**bad) == EINVAL, bad
    assert call(rows=0, g=None) == 0


def test_logprobs(lib):
    size = sz()
    ws = caller(lib.imunpack_logprobs_workspace, [i64, i64, i64, i64, i32, vp], dict(rows=2, vocab=128000, count=1, top=5, dtype=0, out=C.addressof(size)))
    for bad in (dict(rows=-1), dict(rows=1 << 31), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(count=-1), dict(count=1025), dict(top=-1), dict(top=65), dict(vocab=4), dict(dtype=2), dict(out=None)):
        assert ws(**bad) == EINVAL, bad
    assert ws() == 0
    call = caller(lib.imunpack_logprobs, [vp, i64, i64, i64, i32, vp, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, sz, vp],
                  dict(l=FAKE, ldl=128000, rows=2, vocab=128000, dtype=0, t=FAKE, count=1, ignore=-100, top=5, logp=FAKE, lse=FAKE, stats=FAKE, h=FAKE, tl=FAKE, ti=FAKE, ws=FAKE, bytes=1 << 30, st=None))
    for bad in (dict(l=None), dict(ldl=127999), dict(t=None), dict(logp=None), dict(tl=None), dict(ti=None), dict(top=70), dict(count=-2), dict(dtype=9), dict(rows=-1)):
        assert call(**bad) == EINVAL, bad
    assert call(rows=0, l=None) == 0
    if size.value:
        assert call(bytes=size.value - 1) == ESMALL and call(ws=None) == EINVAL and call(ws=FAKE + 4) == EINVAL
    call = caller(lib.imunpack_logprobs_backward, [vp, i64, i64, i64, i32, vp, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, i64, vp],
                  dict(l=FAKE, ldl=50, rows=2, vocab=50, dtype=0, t=FAKE, count=1, ignore=-100, top=2, ti=FAKE, stats=FAKE, h=FAKE, gp=FAKE, gh=FAKE, gt=FAKE, gl=2 * FAKE, ldg=50, st=None))
    for bad in (dict(l=None), dict(ldl=49), dict(ldg=49), dict(t=None), dict(ti=None), dict(stats=None), dict(h=None), dict(gl=None), dict(gl=FAKE, ldg=60), dict(count=2000), dict(vocab=1)):
        assert call(**bad) == EINVAL, bad
    assert call(rows=0, l=None) == 0


def test_column_sums(lib):
    call = caller(lib.imunpack_column_sums, [vp, i64, i64, i64, i32, vp, vp, sz, vp],
                  dict(x=FAKE, ldx=40, rows=5000, cols=40, dtype=0, out=FAKE, ws=FAKE, bytes=1 << 30, st=None))
    for bad in (dict(x=None), dict(ldx=39), dict(rows=-1), dict(rows=(1 << 31) + 1), dict(cols=0), dict(cols=(1 << 24) + 1), dict(dtype=2), dict(out=None), dict(ws=None), dict(ws=FAKE + 8)):
        assert call(**bad) == EINVAL, bad
    assert call(bytes=0) == ESMALL
    bytes_ = sz(7)
    f = lib.imunpack_column_sums_workspace
    f.restype, f.argtypes = i32, [i64, i64, i32, C.POINTER(sz)]
    assert f(100, 40, 0, C.byref(bytes_)) == 0 and bytes_.value == 0
    assert f(5000, 40, 0, C.byref(bytes_)) == 0 and call(bytes=bytes_.value - 1) == ESMALL
    assert f(5000, 40, 0, None) == EINVAL


class Job(C.Structure):
    _fields_ = [("x", vp), ("ldx", i64), ("xs", vp), ("ldxs", i64), ("rows", i64), ("cols", i64), ("dtype", i32), ("square", i32), ("q", vp), ("ldq", i64), ("s", vp), ("lds", i64), ("t", vp), ("ldt", i64),
                ("ts", vp), ("ldts", i64)]


def test_several_tensors(lib):
    f = lib.imunpack_block8_many
    f.restype, f.argtypes = i32, [i32, C.POINTER(Job), i32, vp]
    plain = dict(x=FAKE, ldx=200, rows=300, cols=200, dtype=0, square=0, q=FAKE, ldq=256, s=FAKE, lds=16, t=FAKE, ldt=384, ts=FAKE, ldts=16)
    turn = dict(x=FAKE, ldx=256, xs=FAKE, ldxs=16, rows=300, cols=200, t=FAKE, ldt=384, ts=FAKE, ldts=16)
    def call(first, second, count=2, fmt=0):
        jobs = (Job * 5)(Job(**first), Job(**second))
        return f(count, jobs, fmt, None)
    bads = [{**plain, **c} for c in (dict(x=None), dict(ldx=199), dict(rows=-1), dict(rows=(1 << 31) + 1), dict(rows=(1 << 24) + 1), dict(cols=0), dict(cols=(1 << 24) + 1), dict(dtype=2),
                                     dict(q=None, t=None), dict(q=FAKE + 8), dict(s=None), dict(ldq=255), dict(lds=1), dict(lds=17), dict(t=FAKE + 1), dict(ldt=256), dict(ts=None), dict(ldts=24))]
    bads += [{**turn, **c} for c in (dict(x=None), dict(ldx=200), dict(ldx=255), dict(xs=FAKE + 8), dict(ldxs=1), dict(rows=-1), dict(rows=(1 << 24) + 1), dict(cols=0), dict(t=None), dict(ldt=256),
                                     dict(q=FAKE, ldq=256, s=FAKE, lds=16), dict(square=1))]
    for bad in bads:
        assert call(plain, bad) == EINVAL and call(bad, turn) == EINVAL, bad
    assert call(plain, turn, count=0) == EINVAL and call(plain, turn, count=5) == EINVAL and call(plain, turn, fmt=2) == EINVAL and f(1, None, 0, None) == EINVAL
    assert call({**plain, "rows": 0}, {**turn, "rows": 0}) == 0
