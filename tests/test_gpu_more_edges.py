"""The ends of what the calls on 8-bit tensors and on rows of logits take: powers of two at the ends of their range in every kernel, most tokens and alternatives, more rows than one launch takes,
outputs that nobody asks for."""
import ctypes as C

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def imu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2403_07339_amd import binding
    return binding


@pytest.mark.parametrize("format", ["e4m3", "e5m2"])
@pytest.mark.parametrize("m,n,k", [(5, 40, 200), (70, 130, 200), (500, 300, 1500), (2200, 2100, 256), (64, 64, 9000)])
def test_products_of_the_smallest_and_largest(imu, m, n, k, format):
    """2^-126 by 2^120 (bytes at their lower end, where binary32's exponent has none below): whole numbers times one power of two, exact in every sum."""
    tiny, huge = (imu.imunpack_block8_quantize(torch.full((r, k), v).cuda(), format)[0] for r, v in ((m, 2.0 ** -126), (n, 2.0 ** 120)))
    assert (tiny.scales.view(torch.uint8)[:, : -(-k // 128)] == 0).all()
    for dtype in (torch.float32, torch.bfloat16):
        want = torch.full((m, n), k * 2.0 ** -6).to(dtype).cuda()
        assert torch.equal(imu.imunpack_block8_gemm(tiny, huge, dtype), want)
        assert torch.equal(imu.imunpack_block8_gemm(huge, tiny, dtype), want.t()[:1, :1].expand(n, m))


def test_codes_that_are_nan_in_a_product(imu):
    """They reach the row's or the column's results and no others."""
    for m, n, k in ((7, 50, 300), (90, 130, 600), (700, 520, 256)):
        x, w = torch.randn(m, k).cuda(), torch.randn(n, k).cuda()
        x[3, 5] = float("nan")
        w[11, k - 1] = float("inf")
        a, b = imu.imunpack_block8_quantize(x)[0], imu.imunpack_block8_quantize(w)[0]
        for dtype in (torch.float32, torch.bfloat16):
            bad = torch.isnan(imu.imunpack_block8_gemm(a, b, dtype))
            want = torch.zeros_like(bad)
            want[3], want[:, 11] = True, True
            assert torch.equal(bad, want)


@pytest.mark.parametrize("rows,vocab", [(2, 5000), (2100, 70)])
def test_most_tokens_and_alternatives(imu, rows, vocab):
    """1024 tokens with many twice and 64 alternatives among them.  A gradient's tolerance: 1088 additions in any order, 2^-24 of the magnitudes each, and p within 2^-17."""
    g = torch.Generator().manual_seed(3)
    x = torch.randn(rows, vocab, generator=g) * 2
    t = torch.randint(0, vocab // 2, (rows, 1024), generator=g)
    t[:, 7::50] = -100
    got = imu.imunpack_logprobs(x.cuda(), t.cuda(), top=64)
    logp = torch.log_softmax(x.double(), 1)
    ok = t >= 0
    want = torch.where(ok, logp.gather(1, t.clamp_min(0)), torch.zeros((), dtype=torch.float64))
    assert ((got.logp.cpu().double() - want).abs() <= 2.0 ** -18 + 2.0 ** -22 * want.abs()).all()
    index = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :64]
    assert torch.equal(got.top_index.cpu(), index)
    gp, gt, gh = torch.randn(rows, 1024, generator=g), torch.randn(rows, 64, generator=g), torch.randn(rows, generator=g)
    gl = imu.imunpack_logprobs_backward(x.cuda(), t.cuda(), got, gp.cuda(), gh.cuda(), gt.cuda()).cpu().double()
    w, size = torch.zeros_like(logp), torch.zeros_like(logp)
    for to, by in ((w, lambda v: v), (size, torch.abs)):
        to.scatter_add_(1, t.clamp_min(0), by(gp.double()) * ok)
        to.scatter_add_(1, index, by(gt.double()))
    p = logp.exp()
    h = -(p * logp).sum(1, keepdim=True)
    want = w - p * w.sum(1, keepdim=True) - gh.double()[:, None] * p * (logp + h)
    bound = 1100 * 2.0 ** -24 * (size + p * size.sum(1, keepdim=True)) + 2.0 ** -17 * p * (size.sum(1, keepdim=True) + gh.double().abs()[:, None] * (2 * logp.abs() + 2 * h + 1))
    assert ((gl - want).abs() <= bound + 2.0 ** -23 * want.abs()).all()


def test_no_tokens_to_a_row(imu):
    x = torch.randn(5, 300).cuda()
    none = torch.zeros(5, 0, dtype=torch.int64).cuda()
    got, plain = imu.imunpack_logprobs(x, none, top=2), imu.imunpack_logprobs(x, top=2)
    assert got.logp.shape == (5, 0) and torch.equal(got.lse, plain.lse) and torch.equal(got.top_index, plain.top_index)
    gl = imu.imunpack_logprobs_backward(x, none, got, torch.zeros(5, 0).cuda(), torch.ones(5).cuda())
    assert torch.equal(gl, imu.imunpack_logprobs_backward(x, None, got, None, torch.ones(5).cuda()))
    assert not imu.imunpack_logprobs_backward(x, none, got).any()


def test_outputs_that_nobody_asks_for(imu):
    for rows, vocab in ((3, 900), (2, 60000)):
        x, t = torch.randn(rows, vocab).cuda(), torch.randint(0, vocab, (rows,)).cuda()
        want, ws, logp = imu.imunpack_logprobs(x, t), torch.empty(1 << 20, dtype=torch.uint8, device="cuda"), torch.empty(rows, device="cuda")
        p = lambda v: C.c_void_p(v.data_ptr())  # noqa: E731
        n, i64 = C.c_void_p(None), C.c_int64
        assert imu._lib.imunpack_logprobs(p(x), i64(vocab), i64(rows), i64(vocab), C.c_int(0), p(t), i64(1), i64(-100), i64(0), p(logp), n, n, n, n, n, p(ws), C.c_size_t(1 << 20),
                                          C.c_void_p(imu._stream())) == 0
        assert torch.equal(logp, want.logp)


def test_more_rows_than_a_launch(imu):
    rows = (1 << 22) + 5
    x = torch.randn(rows, 3, device="cuda")
    t = torch.randint(0, 3, (rows,), device="cuda")
    got = imu.imunpack_logprobs(x, t, top=2)
    last = imu.imunpack_logprobs(x[-2500:], t[-2500:], top=2)
    assert all(torch.equal(u[-2500:], v) for u, v in ((got.logp, last.logp), (got.entropy, last.entropy), (got.top_index, last.top_index), (got.top_logp, last.top_logp), (got.stats, last.stats)))
    g = torch.randn(rows, device="cuda")
    gl = imu.imunpack_logprobs_backward(x, t, got, g, g)
    assert torch.equal(gl[-2500:], imu.imunpack_logprobs_backward(x[-2500:], t[-2500:], last, g[-2500:], g[-2500:]))
    assert float((gl.double().sum(1)).abs().max()) < 1e-5     # (a row's gradients add up to nothing)


def test_more_blocks_than_a_launch(imu):
    rows = (1 << 26) + 100
    x = torch.randn(rows, 1, device="cuda", dtype=torch.bfloat16)
    raw = lambda v: v.view(torch.uint8)  # noqa: E731
    for square in (False, True):
        q, _ = imu.imunpack_block8_quantize(x, square=square)
        last, _ = imu.imunpack_block8_quantize(x[-228:], square=square)     # (2^26 is a whole number of squares: the last 228 rows begin with one)
        assert torch.equal(raw(q.codes[-228:]), raw(last.codes)) and torch.equal(raw(q.scales[-228:, :1]), raw(last.scales[:, :1]))
        v = q.values(torch.bfloat16)
        assert torch.equal(v[-228:], last.values(torch.bfloat16)) and bool(((v - x).abs() <= x.abs() / 16 + (2.0 ** -9 if square else 0)).all())
        del q, v
    y, _, kept = imu.imunpack_act8(x, "silu")
    y1, _, k1 = imu.imunpack_act8(x[-228:], "silu")
    assert torch.equal(y[-228:], y1) and torch.equal(raw(kept[0].codes[-228:]), raw(k1[0].codes))
    assert torch.equal(imu.imunpack_act8_backward(y, kept, "silu")[-228:], imu.imunpack_act8_backward(y1, k1, "silu"))
    torch.cuda.empty_cache()
