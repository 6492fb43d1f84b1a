"""The calls around the products reject bad arguments on the host, before the first HIP call (no GPU; the pointers passed are
never dereferenced)."""
import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2403_07339_amd", "libimunpack.so")
EINVAL, ESMALL = -1, -5
vp, i64, i32, f32, f64 = C.c_void_p, C.c_int64, C.c_int, C.c_float, C.c_double
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


def test_rmsnorm(lib):
    call = caller(lib.imunpack_rmsnorm, [vp, i64, vp, i64, vp, i64, i64, i32, i32, f32, vp, i64, vp, i64, vp, vp],
                  dict(x=FAKE, ldx=8, res=FAKE, ldres=8, w=FAKE, rows=2, d=8, dtype=0, wtype=0, eps=1e-6, y=FAKE, ldy=8, h=FAKE, ldh=8, rstd=FAKE, st=None))
    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(ldx=7), dict(ldres=7), dict(ldy=7), dict(ldh=7), dict(rows=-1), dict(d=0), dict(d=(1 << 24) + 1),
                dict(dtype=2), dict(wtype=-1), dict(eps=-1.0), dict(eps=float("nan"))):
        assert call(**bad) == EINVAL, bad
    assert call(rows=0, x=None, y=None, w=None) == 0
    call = caller(lib.imunpack_rmsnorm_quantize, [vp, i64, vp, i64, vp, i64, i64, i32, i32, f32, i32, vp, i64, vp, vp, i64, vp, i64, vp],
                  dict(x=FAKE, ldx=8, res=None, ldres=0, w=FAKE, rows=2, d=8, dtype=1, wtype=0, eps=1e-6, b=8, q=FAKE, ldq=8, scale=FAKE, values=None, ldv=0,
                       h=None, ldh=0, st=None))
    for bad in (dict(b=1), dict(b=9), dict(q=None), dict(scale=None), dict(ldq=7), dict(values=FAKE), dict(h=FAKE), dict(x=None), dict(rows=-1)):
        assert call(**bad) == EINVAL, bad
    assert call(rows=0) == 0


def test_rmsnorm_backward(lib):
    size = C.c_size_t()
    lib.imunpack_rmsnorm_backward_workspace.argtypes = [i64, i64, i32, vp]
    assert lib.imunpack_rmsnorm_backward_workspace(2, 8, 0, None) == EINVAL
    assert lib.imunpack_rmsnorm_backward_workspace(2, 0, 0, C.byref(size)) == EINVAL
    assert lib.imunpack_rmsnorm_backward_workspace(2000, 8, 0, C.byref(size)) == 0 and size.value >= 32
    call = caller(lib.imunpack_rmsnorm_backward, [vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, i64, i64, i32, i32, vp, i64, vp, vp, C.c_size_t, vp],
                  dict(gy=FAKE, ldgy=8, x=FAKE, ldx=8, res=FAKE, ldres=8, gh=FAKE, ldgh=8, w=FAKE, rstd=FAKE, rows=2000, d=8, dtype=0, wtype=0, gx=FAKE, ldgx=8, gw=FAKE,
                       ws=FAKE, bytes=size.value, st=None))
    for bad in (dict(gy=None), dict(x=None), dict(w=None), dict(rstd=None), dict(gx=None), dict(ws=None), dict(ldgy=7), dict(ldx=7), dict(ldres=7), dict(ldgh=7), dict(ldgx=7),
                dict(dtype=5), dict(d=-1), dict(rows=-3)):
        assert call(**bad) == EINVAL, bad
    assert call(bytes=size.value - 1) == ESMALL
    assert call(rows=0, gw=None) == 0


def test_adamw(lib):
    one = (vp * 1)(FAKE)
    none = (vp * 1)(None)
    n = (i64 * 1)(8)
    call = caller(lib.imunpack_adamw, [i64, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, f64, f64, f64, f64, f64, i64, C.c_uint32, vp],
                  dict(count=1, p=one, g=one, m=one, v=one, ms=one, vs=one, copies=None, n=n, gtype=0, bits=8, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=0.0, step=1, seed=0, st=None))
    for bad in (dict(count=-1), dict(p=None), dict(g=None), dict(m=None), dict(v=None), dict(ms=None), dict(vs=None), dict(n=None), dict(p=none), dict(g=none), dict(m=none),
                dict(v=none), dict(ms=none), dict(vs=none), dict(copies=none), dict(n=(i64 * 1)(-1)), dict(gtype=2), dict(bits=16), dict(lr=-1.0), dict(lr=float("inf")),
                dict(b1=1.0), dict(b2=-0.1), dict(eps=float("nan")), dict(wd=-1.0), dict(step=0)):
        assert call(**bad) == EINVAL, bad
    assert call(count=0, p=None, g=None, m=None, v=None, n=None) == 0
    assert call(n=(i64 * 1)(0), p=none, g=none) == 0          # tensors without elements


def test_xent(lib):
    size = C.c_size_t()
    call = caller(lib.imunpack_xent_workspace, [vp, i64, i64, i64, i64, i32, i32, vp], dict(w=FAKE, ldw=64, rows=4, d=64, vocab=100, dtype=0, grad=1, size=C.addressof(size)))
    for bad in (dict(ldw=63), dict(rows=-1), dict(rows=(1 << 22) + 1), dict(d=0), dict(vocab=0), dict(vocab=(1 << 22) + 1), dict(dtype=2), dict(size=None)):
        assert call(**bad) == EINVAL, bad
    assert call(rows=0) == 0 and call(grad=0) == 0
    least = size.value
    assert call() == 0 and size.value > least > 0
    call = caller(lib.imunpack_xent, [vp, i64, vp, i64, vp, i64, i64, i64, i32, i64, i32, vp, vp, vp, i64, vp, i64, vp, C.c_size_t, vp],
                  dict(x=FAKE, ldx=64, w=FAKE, ldw=64, target=FAKE, rows=4, d=64, vocab=100, dtype=0, ignore=-100, how=2, loss=FAKE, grad=None, gx=FAKE, ldgx=64, gw=FAKE, ldgw=64,
                       ws=FAKE, bytes=size.value, st=None))
    for bad in (dict(x=None), dict(w=None), dict(target=None), dict(loss=None, gx=None, gw=None), dict(ws=None), dict(ws=FAKE + 8), dict(ldx=63), dict(ldw=63), dict(ldgx=63),
                dict(ldgw=63), dict(how=3), dict(how=-1), dict(how=0), dict(dtype=-1), dict(d=0), dict(rows=-1), dict(vocab=-5)):
        assert call(**bad) == EINVAL, bad
    assert call(bytes=size.value - 1) == ESMALL
    call = caller(lib.imunpack_xent_rescale, [vp, vp, i64, vp, i64, i32, vp], dict(grad=FAKE, gx=FAKE, nx=4, gw=FAKE, nw=4, dtype=0, st=None))
    for bad in (dict(grad=None), dict(gx=None), dict(gw=None), dict(nx=-1), dict(nw=-1), dict(dtype=3)):
        assert call(**bad) == EINVAL, bad
    assert call(nx=0, nw=0) == 0
