"""Tensors in 8 bits whose powers of two lie at the ends of a byte: turned, and in products by every kernel: codes times such a power are no numbers of bfloat16 (which ends at 2^-133 and below 2^128), and their
products are the contract's all the same.

Tolerances.  One product alone is rounded once, 2^-24 (2^-8) of itself, which is compared as equality with the exact value rounded; what an operand loses below 2^-133 counts at most 2^-126.  Sums of K products:
K 2^-24 of the sum of magnitudes in fp32; bfloat16 results 2^-10 of it and 2^-8 of themselves."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F = torch.float64
FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


@pytest.fixture(scope="module")
def imu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2403_07339_amd import binding
    return binding


def blocks(imu, codes, byte, fmt, behind=127):
    """A Blocks8 of bytes of codes (rows x a multiple of 128) and of powers of two (rows x blocks), `behind` in the places that fill a row of the latter up."""
    scales = torch.full((codes.shape[0], -(-byte.shape[1] // 16) * 16), behind, dtype=torch.uint8)
    scales[:, :byte.shape[1]] = byte
    return imu.Blocks8(codes.cuda().view(FORMATS[fmt]), scales.cuda().view(torch.float8_e8m0fnu), codes.shape[1])


def single(imu, codes, byte, fmt):
    wide = torch.zeros(len(codes), 128, dtype=torch.uint8)
    wide[:, 77] = codes
    return blocks(imu, wide, torch.full((len(codes), 1), byte, dtype=torch.uint8), fmt)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("side", ["few rows", "few rows, B", "tile", "tile, B"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_every_code_at_every_power_of_two(imu, fmt, side, dtype):
    every = torch.arange(256, dtype=torch.uint8)
    v = every.view(FORMATS[fmt]).to(F)
    every, v = every[torch.isfinite(v)], v[torch.isfinite(v)]
    one = torch.full((1 if "few" in side else 40,), int(torch.tensor(1.0).to(torch.float8_e4m3fn).view(torch.uint8)), dtype=torch.uint8)
    for other in (27, 119, 127, 227):
        b = single(imu, one, other, "e4m3")
        for byte in [*range(14), 60, 126, 127, 128, *range(236, 255)]:
            a = single(imu, every, byte, fmt)
            if side == "few rows":
                got = torch.cat([imu.imunpack_block8_gemm(imu.Blocks8(a.codes[k: k + 16], a.scales[k: k + 16], 128), b, dtype) for k in range(0, len(every), 16)])
            else:
                got = imu.imunpack_block8_gemm(b, a, dtype).t() if side.endswith("B") else imu.imunpack_block8_gemm(a, b, dtype)
            want = (v * 2.0 ** (byte - 127) * 2.0 ** (other - 127))[:, None]
            got = got.to(F).cpu()
            near = (got - want).abs() <= 2.0 ** -126
            assert ((got == want.float().to(dtype).to(F)) | near).all(), (other, byte)


# few rows; tiles of 64, alone and in parts; of 128, alone and in parts; of 256 with seventeen blocks
SIZES = [(11, 200, 700), (90, 130, 600), (300, 500, 8192), (700, 5000, 896), (768, 768, 12608), (4000, 3900, 2100)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2")])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_blocks_at_the_ends_among_others(imu, m, n, k, fa, fb, dtype):
    g = torch.Generator().manual_seed(m + n)
    kb = -(-k // 128)

    def operand(rows, fmt):
        x = torch.zeros(rows, kb * 128)
        x[:, :k] = torch.randn(rows, k, generator=g) * (1.0 if fmt == "e4m3" else 2.0)
        codes = x.to(FORMATS[fmt])
        return codes, torch.full((rows, kb), 127, dtype=torch.uint8)

    def in_some(byte, rows, values):   # in one block of each of these rows
        at = torch.randint(0, kb, (len(rows),), generator=g)
        byte[rows, at] = torch.tensor(values, dtype=torch.uint8)[torch.randint(0, len(values), (len(rows),), generator=g)]

    a, sa = operand(m, fa)
    b, sb = operand(n, fb)
    rows = torch.randperm(m, generator=g)
    low, high, mixed = rows[: m // 5], rows[m // 5: 2 * m // 5], rows[2 * m // 5: 3 * m // 5]
    sa[low] = torch.randint(0, 12, (len(low), kb), generator=g).to(torch.uint8)      # whole rows next to 2^-127
    in_some(sa, high, list(range(236, 255)))
    in_some(sa, mixed, list(range(12)))
    cols = torch.randperm(n, generator=g)
    sb[cols[: n // 4]] = 230
    sb[cols[n // 4: n // 2]] = 90
    sb[cols[n // 2: 3 * n // 4]] = torch.randint(0, 12, (3 * n // 4 - n // 2, kb), generator=g).to(torch.uint8)
    value = lambda c, s: c.to(F).cuda().view(c.shape[0], kb, 128).mul(torch.exp2(s.to(F).cuda() - 127)[:, :, None]).view(c.shape)  # noqa: E731
    va, vb = value(a, sa), value(b, sb)
    want, size = va @ vb.t(), va.abs() @ vb.abs().t()
    qa, qb = blocks(imu, a.view(torch.uint8), sa, fa), blocks(imu, b.view(torch.uint8), sb, fb)
    got = imu.imunpack_block8_gemm(qa, qb, dtype)
    fits = size < 2.0 ** 127
    off = (got.to(F) - want).abs()
    limit = k * 2.0 ** -24 * size if dtype == torch.float32 else 2.0 ** -10 * size + 2.0 ** -8 * want.abs()
    assert float(fits.to(F).mean()) > 0.7 and (off[fits] <= limit[fits] + k * 2.0 ** -126).all()
    assert torch.equal(imu.imunpack_block8_gemm(qa, qb, dtype).view(torch.uint8), got.view(torch.uint8))
    bias = torch.randn(n, generator=g).cuda()
    with_bias = imu.imunpack_block8_gemm(qa, qb, torch.float32, bias=bias)
    if dtype == torch.float32:
        assert ((with_bias.to(F) - want - bias.to(F)).abs()[fits] <= ((k + 1) * 2.0 ** -24 * (size + bias.abs().to(F)))[fits] + k * 2.0 ** -126).all()
    # the bytes that fill a row of them up are not looked at
    for behind in (0, 255):
        other = imu.imunpack_block8_gemm(blocks(imu, a.view(torch.uint8), sa, fa, behind), blocks(imu, b.view(torch.uint8), sb, fb, behind), dtype)
        assert torch.equal(other.view(torch.uint8), got.view(torch.uint8))


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_the_largest_values_turned(imu, fmt):
    """Codes of what binary32 has next to 2^128 stand for 2^128, which binary32 has not: turned they are the same values.  No tolerance."""
    from test_gpu_block8 import check_codes, definition
    g = torch.Generator().manual_seed(7)
    x = torch.randn(200, 300, generator=g) * torch.exp2(torch.randint(-140, 120, (1, 300), generator=g).float())
    most = torch.finfo(torch.float32).max
    x[3, 7], x[150, 7], x[5, 200], x[6, 200], x[199, 299], x[8] = most, -most / 3, 1.98 * 2.0 ** 127, 2.0 ** -100, 1.75 * 2.0 ** 127, most
    want, e = definition(x, fmt)
    assert float(want.abs().max()) == 2.0 ** 128
    q, t = imu.imunpack_block8_quantize(x.cuda(), fmt, turned=True)
    check_codes(q, want, e, fmt, 300)
    check_codes(t, *definition(x.t(), fmt), fmt, 200)
    again = definition(want.t(), fmt)
    check_codes(imu.imunpack_block8_turn(q), *again, fmt, 200)
    (_, many), (_, alone) = imu.imunpack_block8_many(q, (x.cuda(), False, False, True), format=fmt)
    check_codes(many, *again, fmt, 200)
    check_codes(alone, *definition(x.t(), fmt), fmt, 200)


@pytest.mark.parametrize("fb", ["e4m3", "e5m2"])
@pytest.mark.parametrize("fa", ["e4m3", "e5m2"])
@pytest.mark.parametrize("rows", [1, 40])
def test_the_least_that_does_not_count(imu, rows, fa, fb):
    """The smallest powers of two beside the largest numbers for which they are left as bfloat16 has them: half a place of 2^-133, 2^-134, times less than 2^8.  And beside the next power of two: rounded once."""
    every = torch.arange(256, dtype=torch.uint8)
    v = every.view(FORMATS[fa]).to(F)
    every, v = every[torch.isfinite(v)], v[torch.isfinite(v)]
    largest = {"e4m3": 448.0, "e5m2": 57344.0}[fb]
    code = int(torch.tensor(largest).to(FORMATS[fb]).view(torch.uint8))
    for other in {"e4m3": (126, 127), "e5m2": (119, 120)}[fb]:
        b = single(imu, torch.full((rows,), code, dtype=torch.uint8), other, fb)
        for byte in range(12):
            a = single(imu, every, byte, fa)
            want = (v * 2.0 ** (byte - 127) * largest * 2.0 ** (other - 127))[None]
            for got in (imu.imunpack_block8_gemm(b, a), imu.imunpack_block8_gemm(a, b).t()):
                off = (got.to(F).cpu() - want).abs()
                assert (off <= 2.0 ** -126).all()
                if largest * 2.0 ** (other - 127) >= 2.0 ** 8:
                    assert (off <= 2.0 ** -24 * want.abs() + 2.0 ** -150).all()
