"""Root-mean-square norm: forward, output in integers, backward, against the formulas in binary64.

Tolerances.  A sum over a row passes at most about 50 binary32 additions on the way of one term (pieces of a thread, the tree over
lanes, the waves), so that statistics are within 50 * 2^-24 and, with the square root's half of it and five more roundings, y
within 64 * 2^-24 of its value (E below).  bfloat16 results are rounded once more: 2^-8 of the value (8 significant bits).  gx subtracts: its
error is measured against the sum of the magnitudes of its terms.  gw: a term passes the rows of a wave, the waves, the partial sums of a
workgroup in 32 and the 32 of those: at most 128 additions for the row counts here."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
E = 64 * 2.0 ** -24
EPS = 1e-6


@pytest.fixture(scope="module")
def imu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2403_07339_amd import binding
    return binding


def data(rows, d, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    x, res, gy, gh = (torch.randn(rows, d, generator=g) for _ in range(4))
    res[:, :: max(1, d // 3)] *= 20.0
    w = 1.0 + 0.3 * torch.randn(d, generator=g)
    to = lambda t: t.to(dtype).cuda()  # noqa: E731
    return to(x), to(res), to(gy), to(gh), w


def round_off(want, dtype):
    return (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24) * want.abs()


def check_forward(imu, x, res, w, y, h, rstd, dtype):
    f = torch.float64
    h64 = x.to(f) + (res.to(f) if res is not None else 0.0)
    r64 = 1.0 / torch.sqrt((h64 * h64).mean(-1, keepdim=True) + EPS)
    y64 = h64 * r64 * w.to(f)
    if res is not None:
        assert ((h.to(f) - h64).abs() <= round_off(h64, dtype) + 2.0 ** -24 * h64.abs()).all()
    assert ((rstd.to(f) - r64[..., 0]).abs() <= E * r64[..., 0]).all()
    assert ((y.to(f) - y64).abs() <= E * y64.abs() + round_off(y64, dtype)).all()


def check_backward(x64, gy, gh, w, gx, gw, dtype):
    f = torch.float64
    h, g, w = x64.reshape(-1, x64.shape[-1]), gy.to(f).reshape(-1, x64.shape[-1]), w.to(f)
    r = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    hat, gyw = h * r, g * w
    back = gh.to(f).reshape(h.shape) if gh is not None else torch.zeros_like(h)
    want = back + r * (gyw - hat * (gyw * hat).mean(1, keepdim=True))
    size = back.abs() + r * (gyw.abs() + hat.abs() * (gyw * hat).abs().mean(1, keepdim=True))
    assert ((gx.to(f).reshape(h.shape) - want).abs() <= E * size + round_off(want, dtype)).all()
    if gw is not None:
        want_w = (g * hat).sum(0)
        assert ((gw.to(f) - want_w).abs() <= 2 * E * (g * hat).abs().sum(0) + (round_off(want_w, gw.dtype))).all()


# rows x d: one element, one row, odd sizes, every way a row is held (a wave, 256 threads, 1024 threads, not at all)
SIZES = [(1, 1), (3, 2), (1, 7), (5, 63), (197, 64), (64, 255), (33, 257), (100, 768), (1000, 1031), (7, 2047), (16, 4096), (9, 5001),
         (3, 8192), (2, 16383), (2, 20000), (3, 40001)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,d", SIZES)
def test_forward_and_backward(imu, rows, d, dtype):
    x, res, gy, gh, w = data(rows, d, dtype, rows + d)
    w = w.to(dtype).cuda()
    y, h, saved = imu.imunpack_rmsnorm(x, w, EPS, residual=res)
    check_forward(imu, x, res, w, y, h, saved.rstd, dtype)
    gx, gw = imu.imunpack_rmsnorm_backward(gy, h, w, saved, gh=gh)
    f = torch.float64
    check_backward(x.to(f) + res.to(f), gy, gh, w, gx, gw, dtype)
    # without a residual, without a gradient of h, without the weight's
    y, h, saved = imu.imunpack_rmsnorm(x, w, EPS)
    assert h is x
    check_forward(imu, x, None, w, y, h, saved.rstd, dtype)
    gx, none = imu.imunpack_rmsnorm_backward(gy, x, w, saved, want_weight=False)
    assert none is None
    check_backward(x.to(f), gy, None, w, gx, None, dtype)
    again, gw = imu.imunpack_rmsnorm_backward(gy, x, w, saved)
    assert torch.equal(again, gx)
    check_backward(x.to(f), gy, None, w, gx, gw, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("b", [8, 4, 2])
@pytest.mark.parametrize("rows,d", [(1, 1), (1, 7), (16, 4096), (50, 1031), (4, 513), (3, 12001), (2, 70000)])
def test_integers_with_a_step_per_row(imu, rows, d, b, dtype):
    x, res, _, _, w = data(rows, d, dtype, 7 * rows + d)
    w, f, top = w.cuda(), torch.float64, 2 ** (b - 1) - 1
    x[0] = -res[0]   # a row of zeros
    q, scale, h, values = imu.imunpack_rmsnorm_quantize(x, w, EPS, b, residual=res, want_values=True)
    h64 = x.to(f) + res.to(f)
    y64 = h64 / torch.sqrt((h64 * h64).mean(1, keepdim=True) + EPS) * w.to(f)
    step = y64.abs().amax(1) / top
    step[0] = 1.0
    assert ((scale.to(f) - step).abs() <= 2 * E * step).all()
    assert q.dtype == torch.int8 and int(q.abs().max()) <= top and not q[0].any()
    want = y64 / scale.to(f)[:, None]
    assert ((q.to(f) - want).abs() <= 0.5 + 2 * E * want.abs()).all()
    v64 = q.to(f) * scale.to(f)[:, None]
    assert ((values.to(f) - v64).abs() <= round_off(v64, dtype)).all()
    assert ((h.to(f) - h64).abs() <= round_off(h64, dtype) + 2.0 ** -24 * h64.abs()).all()
    q2, s2, h2, none = imu.imunpack_rmsnorm_quantize(x, w, EPS, b, residual=res)
    assert none is None and torch.equal(q, q2) and torch.equal(scale, s2) and torch.equal(h, h2)


def test_rows_with_nan_infinity_and_extremes(imu):
    x = torch.randn(6, 300, generator=torch.Generator().manual_seed(1)).cuda()
    w = torch.ones(300, device="cuda")
    x[1, 17], x[2, 299], x[4] = float("nan"), float("inf"), 0.0
    x[5] = 1e-30
    q, scale, _, _ = imu.imunpack_rmsnorm_quantize(x, w, EPS)
    assert torch.isnan(scale[[1, 2]]).all() and not q[1:3].any() and scale[4] == 1.0 and not q[4].any()
    assert torch.isfinite(scale[[0, 3, 5]]).all()
    one, s1, _, _ = imu.imunpack_rmsnorm_quantize(x[[0, 3]], w, EPS)
    assert torch.equal(q[[0, 3]], one) and torch.equal(scale[[0, 3]], s1)     # a bad row does not reach its neighbours
    y, _, saved = imu.imunpack_rmsnorm(x, w, EPS)
    rstd = saved.rstd
    assert torch.isnan(y[1]).all() and not torch.isnan(y[0]).any() and not y[4].any()
    assert abs(float(rstd[4]) - 1000.0) < 1e-3
    y0, _, _ = imu.imunpack_rmsnorm(torch.zeros(2, 5, device="cuda"), torch.ones(5, device="cuda"), 0.0)
    assert torch.isnan(y0).all()   # 0 / 0, as the formula has it


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_leading_dimensions_and_empty_inputs(imu, dtype):
    x, res, gy, gh, w = data(24, 130, dtype, 3)
    w = w.cuda()
    want = imu.imunpack_rmsnorm(x, w, EPS, residual=res)
    back = imu.imunpack_rmsnorm_backward(gy, want[1], w, want[2], gh=gh)
    wide = lambda t: torch.cat([t, t, t], 1)[:, 130:260]  # noqa: E731  (rows 390 apart, at addresses that are not multiples of 16)
    got = imu.imunpack_rmsnorm(wide(x), w, EPS, residual=res.t().contiguous().t())
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[2].rstd, want[2].rstd)
    got = imu.imunpack_rmsnorm_backward(wide(gy), wide(want[1]), w, imu.NormSaved(want[2].rstd, wide(x), wide(res)), gh=wide(gh))
    assert all(torch.equal(a, b) for a, b in zip(got, back))
    got = imu.imunpack_rmsnorm(x.view(2, 3, 4, 130).transpose(0, 2), w, EPS, residual=res.view(2, 3, 4, 130).transpose(0, 2))
    assert torch.equal(got[0], want[0].view(2, 3, 4, 130).transpose(0, 2))
    same = x[:1].expand(24, 130)
    assert torch.equal(imu.imunpack_rmsnorm(same, w, EPS)[0], imu.imunpack_rmsnorm(same.contiguous(), w, EPS)[0])
    y, h, saved = imu.imunpack_rmsnorm(x[:0], w, EPS, residual=res[:0])
    assert y.shape == (0, 130) and saved.rstd.shape == (0,)
    gx, gw = imu.imunpack_rmsnorm_backward(gy[:0], h, w, saved)
    assert gx.shape == (0, 130) and not gw.any()
    q, scale, _, _ = imu.imunpack_rmsnorm_quantize(x[:0], w, EPS)
    assert q.shape == (0, 130) and scale.shape == (0,)


def test_rows_further_apart_than_32_bits(imu):
    pitch = (1 << 31) + 8
    flat = torch.empty(pitch + 64, dtype=torch.bfloat16, device="cuda")
    x = flat.as_strided((2, 64), (pitch, 1))
    x.copy_(torch.randn(2, 64, generator=torch.Generator().manual_seed(2)))
    w = torch.ones(64, device="cuda")
    assert torch.equal(imu.imunpack_rmsnorm(x, w, EPS)[0], imu.imunpack_rmsnorm(x.contiguous(), w, EPS)[0])


def test_another_stream_and_a_graph(imu):
    x, res, gy, gh, w = data(300, 768, torch.float32, 5)
    w = w.cuda()
    want = imu.imunpack_rmsnorm(x, w, EPS, residual=res)
    back = imu.imunpack_rmsnorm_backward(gy, want[1], w, want[2], gh=gh)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y, h, rstd = imu.imunpack_rmsnorm(x, w, EPS, residual=res)
        gx, gw = imu.imunpack_rmsnorm_backward(gy, h, w, rstd, gh=gh)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, want[0]) and torch.equal(gx, back[0]) and torch.equal(gw, back[1])
    xs = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, h, rstd = imu.imunpack_rmsnorm(xs, w, EPS, residual=res)
        gx, gw = imu.imunpack_rmsnorm_backward(gy, h, w, rstd, gh=gh)
    for k in range(3):
        xs.copy_(x * (k + 1))
        graph.replay()
        e = imu.imunpack_rmsnorm(xs, w, EPS, residual=res)
        torch.cuda.synchronize()
        assert torch.equal(y, e[0]) and all(torch.equal(a, b) for a, b in zip((gx, gw), imu.imunpack_rmsnorm_backward(gy, e[1], w, e[2], gh=gh)))


def test_module_gradients_against_autograd_and_differences(imu):
    from paper_2403_07339_amd import norm
    x, res, gy, gh, _ = data(40, 96, torch.float32, 9)
    layer = norm.RMSNorm(96, EPS, device="cuda")
    with torch.no_grad():
        layer.weight.copy_(torch.linspace(0.5, 1.5, 96))
    x.requires_grad_()
    res.requires_grad_()
    y, h = layer(x, res)
    torch.autograd.backward([y, h], [gy, gh])
    f = torch.float64
    x6, r6, w6 = (t.detach().to(f).requires_grad_() for t in (x, res, layer.weight))
    h6 = x6 + r6
    y6 = h6 / torch.sqrt((h6 * h6).mean(1, keepdim=True) + EPS) * w6
    torch.autograd.backward([y6, h6], [gy.to(f), gh.to(f)])
    for got, want in ((x.grad, x6.grad), (res.grad, r6.grad), (layer.weight.grad, w6.grad)):
        assert float((got.to(f) - want).norm() / want.norm()) < 2 * E
    # central differences of the kernel's own forward pass along a random direction: truncation t^2 / 6 times a third derivative of
    # order one, rounding 2^-24 / t of a sum of order sqrt(size): both below 2e-3 of the slope's scale for t = 1/64
    way, t = torch.randn(40, 96, generator=torch.Generator().manual_seed(4)).cuda(), 1.0 / 64
    def value(at):
        y, h, _ = imu.imunpack_rmsnorm(at, layer.weight.detach(), EPS, residual=res.detach())
        return float((y.to(f) * gy.to(f)).sum() + (h.to(f) * gh.to(f)).sum())
    slope = (value(x.detach() + t * way) - value(x.detach() - t * way)) / (2 * t)
    assert abs(slope - float((x.grad.to(f) * way.to(f)).sum())) < 2e-3 * float(x.grad.norm() * way.norm())
    # only one of the two outputs is used
    x.grad = None
    y, h = layer(x, res.detach())
    y.backward(gy)
    only = x.grad.clone()
    x.grad = None
    y, h = layer(x, res.detach())
    h.backward(gh)
    assert torch.equal(x.grad, gh)
    assert float((only + gh - x6.grad).norm() / x6.grad.norm()) < 1e-5


def test_integers_go_through_the_exact_product(imu):
    """The integers of the norm as the first operand of the exact product: In-Bound, so their rows and columns are not split."""
    g = torch.Generator().manual_seed(11)
    x = torch.randn(64, 192, generator=g).cuda()
    x[:, 3] *= 60.0
    w = torch.randn(80, 192, generator=g).cuda()
    w[torch.rand(80, 192, generator=g).cuda() < 0.01] *= 64.0
    q, scale, _, _ = imu.imunpack_rmsnorm_quantize(x, torch.ones(192, device="cuda"), EPS, b=8)
    step = float(w.std() * 4 / 127)
    Qw, _, _ = imu.imunpack_quantize(w, step, 8)
    Qa = q.to(torch.int32)
    plan = imu.imunpack_plan(Qa, Qw, 8, imu.BOTH, imu.BOTH)
    assert plan.dims()[0] == 64
    a, b = imu.imunpack_unpack(plan, Qa, Qw)
    out = torch.empty(64, 80, dtype=torch.int64, device="cuda")
    imu.imunpack_gemm(plan, a, b, 1.0, step, out, None)
    assert np.array_equal(out.cpu().numpy(), Qa.cpu().numpy().astype(np.int64) @ Qw.cpu().numpy().astype(np.int64).T)


def test_refusals(imu):
    x, w = torch.zeros(4, 8, device="cuda"), torch.ones(8, device="cuda")
    with pytest.raises(ValueError):
        imu.imunpack_rmsnorm(x.half(), w)
    with pytest.raises(ValueError):
        imu.imunpack_rmsnorm(x, w[:7])
    with pytest.raises(ValueError):
        imu.imunpack_rmsnorm(x, w, residual=x.bfloat16())
    with pytest.raises(ValueError):
        imu.imunpack_rmsnorm(x.cpu(), w)
    with pytest.raises(imu.ImunpackError):
        imu.imunpack_rmsnorm(x, w, eps=-1.0)
    with pytest.raises(imu.ImunpackError):
        imu.imunpack_rmsnorm_quantize(x, w, b=9)
    with pytest.raises(ValueError):
        imu.imunpack_rmsnorm_backward(x, x.bfloat16(), w, imu.NormSaved(torch.ones(4, device="cuda")))
    with pytest.raises(ValueError):
        imu.imunpack_rmsnorm_backward(x, x, w, imu.NormSaved(torch.ones(3, device="cuda")))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,d", [(1, 64), (37, 1031), (200, 5000), (256, 768), (257, 768), (40, 20000)])
def test_gradient_in_the_place_of_what_it_is_made_from(imu, rows, d, dtype):
    """gx may be gy or gh (the entry point in C; the binding gives it memory of its own): the same bits as elsewhere, up to 256 rows and beyond."""
    import ctypes as C
    x, res, gy, gh, w = data(rows, d, dtype, rows + 2 * d)
    w = w.cuda()
    _, _, saved = imu.imunpack_rmsnorm(x, w, EPS, residual=res)
    t, size = 1 if dtype == torch.bfloat16 else 0, C.c_size_t()
    assert imu._lib.imunpack_rmsnorm_backward_workspace(rows, d, t, C.byref(size)) == 0
    ws = torch.empty(size.value, dtype=torch.uint8, device="cuda")

    def call(gy, gh, gx):
        gw = torch.full((d,), 7.0, device="cuda")
        assert imu._lib.imunpack_rmsnorm_backward(gy.data_ptr(), d, x.data_ptr(), d, res.data_ptr(), d, gh.data_ptr(), d, w.data_ptr(), saved.rstd.data_ptr(), rows, d, t, 0,
                                                  gx.data_ptr(), d, gw.data_ptr(), ws.data_ptr(), size.value, imu._stream()) == 0
        return gx, gw

    want = call(gy, gh, torch.empty_like(gy))
    check_backward(x.to(torch.float64) + res.to(torch.float64), gy, gh, w, want[0], want[1], dtype)
    for _ in range(5):
        at = gy.clone()
        got = call(at, gh, at)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        at = gh.clone()
        got = call(gy, at, at)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("b", [8, 4, 2])
def test_integers_of_next_to_nothing_are_in_bound(imu, b):
    """y of 2 to 800 times 2^-149: rows with one element (their 1 / rms is exactly 2), weights of a few steps of binary32 below 2^-126."""
    top, f = 2 ** (b - 1) - 1, torch.float64
    x = torch.eye(4, device="cuda")
    for first in range(1, 401, 4):
        w = torch.arange(first, first + 4, dtype=torch.int32, device="cuda").view(torch.float32)
        q, scale, _, values = imu.imunpack_rmsnorm_quantize(x, w, 0.0, b, want_values=True)
        y = torch.diag(2.0 * w.to(f))
        assert int(q.abs().max()) <= top and (torch.diag(q) != 0).all()
        assert ((q.to(f) * scale.to(f)[:, None] - y).abs() <= 0.5 * scale.to(f)[:, None]).all()
        assert torch.equal(values.to(f), q.to(f) * scale.to(f)[:, None])
