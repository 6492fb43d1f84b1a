"""Tensors in 8-bit floating point with a power of two per block, their products, activations kept that way: against the definitions in binary64.

Tolerances.  Codes and scales have none: x 2^-e is exact and rounded once, so they are compared bit for bit.  A product whose operands are small whole
numbers (times powers of two that are the same along the contraction) has exact sums in binary32, and its results are compared bit for bit too (bfloat16: with
the sum rounded once).  Others: fp32 results pass at most one rounding to binary32 a place of the contraction, K 2^-24 of the sum of magnitudes (and one for the bias);
bfloat16 results may come from a matrix instruction that cuts each of eight products it adds below 2^-13 of the largest of them, so 8 * 2^-13 = 2^-10 of the sum of
magnitudes at most, and are rounded by 2^-8 of themselves.
Activations: f(u) is three to five binary32 operations behind exp or erf, each of which is within 2^-22 here: 16 * 2^-24 of |u| (|f| <= |u|), gated times the other factor; slopes
are within 16 * 2^-24 of 1.2."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
E = 16 * 2.0 ** -24
F = torch.float64
TOP = {"e4m3": (448.0, 3, -6), "e5m2": (57344.0, 2, -14)}
CODE = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


@pytest.fixture(scope="module")
def imu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2403_07339_amd import binding
    return binding


def definition(x, fmt, square=False):
    """(values, exponents per element) of a matrix, in binary64 on the host."""
    x = x.detach().double().cpu()
    rows, cols = x.shape
    top, bits, least = TOP[fmt]
    pad = torch.zeros(-(-rows // 128) * 128 if square else rows, -(-cols // 128) * 128, dtype=F)
    pad[:rows, :cols] = x
    tall = 128 if square else 1
    b = pad.view(pad.shape[0] // tall, tall, pad.shape[1] // 128, 128)
    size = torch.where(torch.isfinite(b), b.abs(), torch.zeros((), dtype=F)).amax((1, 3), keepdim=True)
    m, e = np.frexp((size / top).numpy())    # size / top = m 2^e, m in [0.5, 1): 2^(e - 1) only where m is 0.5 (a quotient by 7 2^k is not rounded onto 0.5)
    e = torch.from_numpy(np.where(size.numpy() == 0, 0, np.maximum(np.where(m == 0.5, e - 1, e), -127)).astype(np.float64))
    v = b * torch.exp2(-e)
    grain = torch.exp2(torch.floor(torch.log2(v.abs().clamp(2.0 ** least, top))) - bits)
    v = torch.round(v / grain) * grain * torch.exp2(e)
    full = lambda t: t.expand(b.shape).reshape(pad.shape)[:rows]  # noqa: E731
    return full(v)[:, :cols], full(e)[:, ::128].contiguous()


def exponents(q):
    return q.scales.view(torch.uint8).cpu().double()[:, : q.codes.shape[1] // 128] - 127


def check_codes(q, want, e, fmt, cols):
    assert q.cols == cols and q.codes.dtype == CODE[fmt] and q.codes.shape[0] == want.shape[0]
    assert torch.equal(exponents(q), e)
    got = q.codes.to(torch.float32).double().cpu() * torch.exp2(e).repeat_interleave(128, 1)
    assert torch.equal(got[:, :cols].nan_to_num(nan=-7.0), want.nan_to_num(nan=-7.0)), (got[:, :cols] - want).abs().max()
    assert not q.codes.view(torch.uint8)[:, cols:].any()


def matrix(rows, cols, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(3 * torch.randn(rows, 1, generator=g))
    x[:, ::37] *= 50.0
    x[rows // 2, : min(cols, 130)] = 0.0
    return x.to(dtype).cuda()


SIZES = [(1, 1), (1, 128), (3, 127), (2, 129), (128, 128), (130, 300), (197, 256), (1000, 1031), (16, 4096), (5, 20000), (257, 128)]


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_codes_and_scales(imu, rows, cols, dtype, fmt):
    x = matrix(rows, cols, dtype, rows + cols)
    want, e = definition(x, fmt)
    t_want, t_e = definition(x.t(), fmt)
    q, none = imu.imunpack_block8_quantize(x, fmt)
    assert none is None
    check_codes(q, want, e, fmt, cols)
    q, t = imu.imunpack_block8_quantize(x, fmt, turned=True)
    check_codes(q, want, e, fmt, cols)
    check_codes(t, t_want, t_e, fmt, rows)
    none, t = imu.imunpack_block8_quantize(x, fmt, turned=True, lying=False)
    assert none is None
    check_codes(t, t_want, t_e, fmt, rows)
    # what is in 8 bits already, turned: its values, in blocks along the columns
    again = imu.imunpack_block8_turn(q)
    check_codes(again, *definition(want.t(), fmt), fmt, rows)
    # square blocks, both ways: one set of values
    want, e = definition(x, fmt, True)
    q, t = imu.imunpack_block8_quantize(x, fmt, square=True, turned=True)
    check_codes(q, want, e, fmt, cols)
    t_values, t_e = definition(x.t(), fmt, True)
    assert torch.equal(t_values, want.t())
    check_codes(t, t_values, t_e, fmt, rows)
    q, _ = imu.imunpack_block8_quantize(x, fmt, square=True)
    check_codes(q, want, e, fmt, cols)
    assert torch.equal(q.values().double().cpu(), want)
    assert torch.equal(q.values(torch.bfloat16).double().cpu(), want)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_every_edge_of_the_scale(imu, fmt):
    """Largest magnitudes next to top 2^e, of every exponent binary32 has, its subnormals among them; every code's ties."""
    top = TOP[fmt][0]
    rows = []
    for k in range(-149, 128):
        for f in (1.0, 1.75, 1.75 * (1 + 2.0 ** -23), 1.75 * (1 - 2.0 ** -24), 2 - 2.0 ** -23):
            v = np.float32(f * 2.0 ** k) if f * 2.0 ** k < 2.0 ** 128 else np.float32(0)
            rows.append(torch.tensor([float(v), float(v) / 3, -float(v) * 2.0 ** -17, float(v) * 2.0 ** -9]))
    x = torch.stack(rows).float()
    ties = torch.arange(0, 128, dtype=torch.float32).repeat(2, 1)   # all codes of e4m3 from 0 on, and halfway to the next
    every = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    ties = torch.cat([every, (every[1:] + every[:-1]) / 2]).repeat(3, 1) * torch.tensor([[1.0], [-1.0], [2.0 ** -20]])
    for y in (x, ties):
        q, _ = imu.imunpack_block8_quantize(y.cuda(), fmt)
        want, e = definition(y, fmt)
        check_codes(q, want, e, fmt, y.shape[1])
    assert top in (448.0, 57344.0)


def test_infinity_and_nan_cost_their_neighbours_nothing(imu):
    x = torch.randn(130, 260)
    clean, e = definition(x, "e4m3")
    bad = x.clone()
    bad[3, 5], bad[7, 200], bad[9, 131] = float("inf"), float("nan"), -float("inf")
    ref = x.clone()
    ref[3, 5] = ref[7, 200] = ref[9, 131] = 0.0
    want, e = definition(ref, "e4m3")
    for q in (imu.imunpack_block8_quantize(bad.cuda())[0], imu.imunpack_block8_quantize(bad.cuda(), turned=True)[0]):
        assert torch.equal(exponents(q), e)
        got = q.values().cpu().double()
        assert torch.isnan(got[3, 5]) and torch.isnan(got[7, 200]) and torch.isnan(got[9, 131])
        got[3, 5] = got[7, 200] = got[9, 131] = 0.0
        assert torch.equal(got, want)
    q5, _ = imu.imunpack_block8_quantize(bad.cuda(), "e5m2")
    got = q5.values()
    assert torch.isinf(got[3, 5]) and torch.isnan(got[7, 200]) and torch.isinf(got[9, 131]) and torch.isfinite(got).sum() == x.numel() - 3
    y = imu.imunpack_block8_gemm(imu.imunpack_block8_quantize(bad.cuda())[0], imu.imunpack_block8_quantize(x.cuda())[0])
    rows = torch.isnan(y).any(1).nonzero()[:, 0].tolist()
    assert rows == [3, 7, 9] and torch.isnan(y[rows]).all()
    y = imu.imunpack_block8_gemm(imu.imunpack_block8_quantize(bad.cuda())[0], imu.imunpack_block8_quantize(x.cuda())[0], torch.bfloat16)
    assert torch.isnan(y).any(1).nonzero()[:, 0].tolist() == rows


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_layouts_of_x(imu, dtype):
    base = matrix(400, 700, dtype, 3)
    for x in (base[5:105, 3:260], base[::2, :300], base.t()[10:200, :333], base[:1].expand(70, 700), base[:, :1], base.view(40, 10, 700), base[7], base[:0]):
        flat = x.reshape(-1, x.shape[-1])
        want, e = definition(flat, "e4m3")
        q, t = imu.imunpack_block8_quantize(x, turned=x.numel() > 0)
        check_codes(q, want, e, "e4m3", x.shape[-1])
        if t is not None:
            check_codes(t, *definition(flat.t(), "e4m3"), "e4m3", flat.shape[0])


# ---- products ------------------------------------------------------------------------------------------
def whole_numbers(rows, cols, fmt, seed, up=0):
    """A Blocks8-able matrix of whole numbers -7 .. 7 (e5m2: what it has of them), every block's largest 7 so that its scale is known, rows times powers of two."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randint(-7, 8, (rows, cols), generator=g).float()
    if fmt == "e5m2":
        x = x.to(CODE[fmt]).float()
    return x * torch.exp2(torch.randint(-up, up + 1, (rows, 1), generator=g).float()) if up else x


GEMMS = [(1, 1, 1), (1, 64, 128), (2, 3, 129), (16, 4096, 256), (17, 100, 300), (33, 777, 1031), (64, 64, 64), (65, 129, 4096), (100, 1000, 256), (128, 128, 127),
         (197, 1000, 256), (256, 256, 384), (300, 520, 2048), (512, 768, 768), (1000, 777, 1031), (1031, 1000, 777), (2048, 2304, 640), (4096, 1111, 512), (5000, 2600, 200)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("m,n,k", GEMMS)
def test_products_of_whole_numbers_are_exact(imu, m, n, k, fa, fb, dtype):
    if (fa, fb) in (("e4m3", "e5m2"), ("e5m2", "e5m2")) and m * n > 300000:
        pytest.skip("two formats at the smaller sizes")
    a, b = whole_numbers(m, k, fa, m + n + k, 5), whole_numbers(n, k, fb, m * n + k, 5)
    bias = torch.randint(-100, 101, (n,)).float()
    want = a.cuda().double() @ b.cuda().double().t()
    qa, qb = imu.imunpack_block8_quantize(a.cuda(), fa)[0], imu.imunpack_block8_quantize(b.cuda(), fb)[0]
    got = imu.imunpack_block8_gemm(qa, qb, dtype)
    assert got.dtype == dtype and got.shape == (m, n)
    assert torch.equal(got, want.float().to(dtype))
    got = imu.imunpack_block8_gemm(qa, qb, dtype, bias=bias.cuda())
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    full = want + bias.cuda().double()
    assert ((got.double() - full).abs() <= step * full.abs() + 2.0 ** -24 * want.abs()).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", [(1, 50, 700), (16, 4096, 4096), (60, 300, 3000), (197, 1000, 256), (300, 500, 8192), (1000, 777, 1031), (2048, 2048, 2048), (700, 5000, 896)])
def test_products(imu, m, n, k, dtype):
    a, b = matrix(m, k, torch.float32, m).cpu(), matrix(n, k, torch.float32, n + 1).cpu()
    b /= b.abs().amax(1, keepdim=True).clamp_min(1e-20)
    for fa, square in (("e4m3", False), ("e5m2", True)):
        qa, qb = imu.imunpack_block8_quantize(a.cuda(), fa)[0], imu.imunpack_block8_quantize(b.cuda(), "e4m3", square=square)[0]
        va, vb = qa.values().double(), qb.values().double()
        want, size = va @ vb.t(), va.abs() @ vb.abs().t()
        got = imu.imunpack_block8_gemm(qa, qb, dtype).double()
        off = (got - want).abs()
        if dtype == torch.float32:
            assert (off <= k * 2.0 ** -24 * size).all()
            assert (got - want).norm() <= 2e-6 * want.norm()
        else:
            assert (off <= 2.0 ** -10 * size + 2.0 ** -8 * want.abs()).all()
            assert (got - want).norm() <= 2.0 ** -8 * want.norm()
        assert torch.equal(imu.imunpack_block8_gemm(qa, qb, dtype).double(), got)   # the same bits again


def test_scales_of_every_size_in_a_product(imu):
    """Blocks whose powers of two lie far apart, in every place of the groups that a kernel takes them in."""
    k = 128 * 37
    a, b = torch.ones(40, k), torch.ones(70, k)
    up = torch.arange(37).float() - 18
    a *= torch.exp2(3 * up).repeat_interleave(128)
    b *= torch.exp2(-3 * up + (torch.arange(37) % 3).float()).repeat_interleave(128)
    want = (a.double() @ b.double().t()).cuda()
    qa, qb = (imu.imunpack_block8_quantize(t.cuda())[0] for t in (a, b))
    assert torch.equal(imu.imunpack_block8_gemm(qa, qb).double(), want)
    assert torch.equal(imu.imunpack_block8_gemm(qa, qb, torch.bfloat16), want.float().bfloat16())
    tiny, huge = (imu.imunpack_block8_quantize(torch.full((5, 200), v).cuda())[0] for v in (2.0 ** -126, 2.0 ** 120))
    got = imu.imunpack_block8_gemm(tiny, huge)
    assert torch.equal(got, torch.full((5, 5), 200 * 2.0 ** -6).cuda())


def test_a_product_of_views_and_streams_and_graphs(imu):
    a, b = matrix(300, 500, torch.float32, 1), matrix(200, 500, torch.float32, 2)
    qa, qb = imu.imunpack_block8_quantize(a)[0], imu.imunpack_block8_quantize(b)[0]
    want = imu.imunpack_block8_gemm(qa, qb)
    rows = imu.Blocks8(qa.codes[17:117], qa.scales[17:117], 500)
    assert torch.equal(imu.imunpack_block8_gemm(rows, qb), want[17:117])
    every = imu.Blocks8(qa.codes[::3], qa.scales[::3], 500)
    assert torch.equal(imu.imunpack_block8_gemm(every, qb), want[::3])
    assert torch.equal(imu.imunpack_block8_gemm(imu.Blocks8(qa.codes[:0], qa.scales[:0], 500), qb), want[:0])
    assert torch.equal(imu.imunpack_block8_gemm(qa, imu.Blocks8(qb.codes[5:6], qb.scales[5:6], 500)), want[:, 5:6])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = imu.imunpack_block8_gemm(qa, qb)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(other, want)
    # the whole chain in a graph, replayed with other inputs
    x = a.clone()
    def chain():
        q, t = imu.imunpack_block8_quantize(x, turned=True)
        return imu.imunpack_block8_gemm(q, qb), imu.imunpack_block8_gemm(t, imu.imunpack_block8_turn(q))
    chain()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = chain()
    for k in range(4):
        x.copy_(a * (k + 1) ** 3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(out, chain()))


def test_refusals_of_products(imu):
    q = imu.imunpack_block8_quantize(matrix(10, 200, torch.float32))[0]
    good = dict(codes=q.codes, scales=q.scales, cols=200)
    for bad in (dict(codes=q.codes[:, :200]), dict(cols=257), dict(scales=q.scales[:, :2]), dict(scales=q.scales[:9]), dict(codes=q.codes.view(torch.uint8)),
                dict(scales=q.scales.view(torch.uint8)), dict(codes=q.codes.cpu()), dict(codes=q.codes.t()), dict(cols=0), dict(codes=q.codes[:, 1:])):
        with pytest.raises(ValueError):
            imu.imunpack_block8_gemm(imu.Blocks8(**{**good, **bad}), q)
        with pytest.raises(ValueError):
            imu.imunpack_block8_turn(imu.Blocks8(**{**good, **bad}))
    with pytest.raises(ValueError):
        imu.imunpack_block8_gemm(q, imu.imunpack_block8_quantize(matrix(10, 201, torch.float32))[0])
    with pytest.raises(ValueError):
        imu.imunpack_block8_gemm(q, q, torch.float16)
    for bias in (torch.zeros(9).cuda(), torch.zeros(10).cuda().bfloat16(), torch.zeros(10), torch.zeros(20).cuda()[::2]):
        with pytest.raises(ValueError):
            imu.imunpack_block8_gemm(q, q, bias=bias)
    for bad in (torch.zeros(3, 4).cuda().half(), torch.zeros(3, 4), torch.zeros(3, 0).cuda(), torch.zeros(()).cuda()):
        with pytest.raises(ValueError):
            imu.imunpack_block8_quantize(bad)
    with pytest.raises(ValueError):
        imu.imunpack_block8_quantize(torch.zeros(3, 4).cuda(), "e3m4")
    with pytest.raises(ValueError):
        imu.imunpack_block8_quantize(torch.zeros(3, 4).cuda(), lying=False)
    with pytest.raises(ValueError):
        imu.imunpack_block8_quantize(torch.zeros(0, 4).cuda(), turned=True)


# ---- activations ---------------------------------------------------------------------------------------
def act64(u, act):
    return u * torch.special.ndtr(u) if act == "gelu" else u * torch.sigmoid(u)


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 127), (5, 128), (2, 257), (197, 256), (100, 1031), (1, 11008), (64, 4096)])
def test_activations(imu, rows, cols, dtype, gated, act):
    g = torch.Generator().manual_seed(rows + cols)
    u = torch.randn(rows, cols * (2 if gated else 1), generator=g) * 2
    u[:, ::19] *= 10.0
    u, gy = u.to(dtype).cuda(), torch.randn(rows, cols, generator=g).to(dtype).cuda()
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    parts = list(u.double().split(cols, 1))
    want = act64(parts[0], act) * (parts[1] if gated else 1.0)
    size = parts[0].abs() * (parts[1].abs() if gated else 1.0)
    y, codes, kept = imu.imunpack_act8(u, act, gated)
    assert codes is None and len(kept) == (2 if gated else 1)
    assert ((y.double() - want).abs() <= E * size + step * want.abs()).all()
    for part, k in zip(parts, kept):
        check_codes(k, *definition(part, "e4m3"), "e4m3", cols)
    # the gradient, of the values that were kept
    values = [k.values().double().requires_grad_() for k in kept]
    (act64(values[0], act) * (values[1] if gated else 1.0)).backward(gy.double())
    want_g = torch.cat([v.grad for v in values], 1)
    other = torch.cat([values[1].detach().abs(), values[0].detach().abs()], 1) if gated else torch.ones_like(want_g)
    gu = imu.imunpack_act8_backward(gy, kept, act, gated)
    size_g = 1.2 * other * gy.double().abs().repeat(1, 2 if gated else 1)
    assert gu.dtype == dtype and gu.shape == u.shape
    assert ((gu.double() - want_g).abs() <= E * size_g + step * want_g.abs() + 2.0 ** -140).all()
    # its result in 8 bits: the codes of a value that binary32 has next to the exact one, and their values in dtype
    y8, codes, none = imu.imunpack_act8(u, act, gated, quantize=True, keep=False)
    assert none is None
    v = codes.values().double()
    top = size.abs().amax()
    scale = torch.exp2(exponents(codes)).repeat_interleave(128, 1)[:, :cols].cuda()
    assert ((v - want).abs() <= (2.0 ** -4 + E) * want.abs() + 2.0 ** -10 * scale + E * size).all()
    assert ((want.abs() <= 448.0 * scale * (1 + E) + E * size)).all() and top >= 0
    assert torch.equal(y8.double(), v.to(dtype).double())
    none, only, _ = imu.imunpack_act8(u, act, gated, quantize=True, want_y=False)
    assert none is None and torch.equal(only.codes.view(torch.uint8), codes.codes.view(torch.uint8)) and torch.equal(exponents(only), exponents(codes))


def test_gradient_of_an_activation_against_differences(imu):
    for act in ("gelu", "silu"):
        v = torch.linspace(-6, 6, 97).to(torch.float8_e4m3fn).float().cuda()[None]   # numbers that 8 bits hold
        _, _, kept = imu.imunpack_act8(v, act)
        assert torch.equal(kept[0].values(), v)
        gu = imu.imunpack_act8_backward(torch.ones_like(v), kept, act).double()
        d = 1e-5
        slope = (act64(v.double() + d, act) - act64(v.double() - d, act)) / (2 * d)   # (error d^2 / 6 times a third derivative below 2: 4e-11, and 1e-16 / d)
        assert ((gu - slope).abs() <= 1.2 * E + 1e-10).all()


def test_layouts_and_refusals_of_activations(imu):
    base = torch.randn(60, 600).cuda()
    whole, _, _ = imu.imunpack_act8(base[3:33, 5:405].contiguous(), "silu", True)
    part, _, kept = imu.imunpack_act8(base[3:33, 5:405], "silu", True)
    assert torch.equal(whole, part)
    turned, _, _ = imu.imunpack_act8(base.t()[:, :50], "gelu")
    assert torch.equal(turned, imu.imunpack_act8(base.t()[:, :50].contiguous(), "gelu")[0])
    deep, _, k3 = imu.imunpack_act8(base.view(6, 10, 600), "gelu")
    assert deep.shape == (6, 10, 600)
    g = torch.randn(6, 10, 600).cuda()
    assert imu.imunpack_act8_backward(g, k3, "gelu").shape == (6, 10, 600)
    one = torch.ones((), device="cuda").expand(30, 200)   # the gradient of a sum
    assert torch.equal(imu.imunpack_act8_backward(one, kept, "silu", True), imu.imunpack_act8_backward(one.contiguous(), kept, "silu", True))
    empty, _, k0 = imu.imunpack_act8(base[:0], "gelu")
    assert empty.shape == (0, 600) and imu.imunpack_act8_backward(base[:0], k0, "gelu").shape == (0, 600)
    for call in (lambda: imu.imunpack_act8(base[:, :5], "gelu", True), lambda: imu.imunpack_act8(base, "relu"), lambda: imu.imunpack_act8(base.half()), lambda: imu.imunpack_act8(base.cpu()),
                 lambda: imu.imunpack_act8(base, want_y=False), lambda: imu.imunpack_act8_backward(base, kept, "silu", True), lambda: imu.imunpack_act8_backward(base[:30, :200], kept, "silu"),
                 lambda: imu.imunpack_act8_backward(base[:30, :200].cpu(), kept, "silu", True), lambda: imu.imunpack_act8_backward(base[:30, :200], None)):
        with pytest.raises(ValueError):
            call()
