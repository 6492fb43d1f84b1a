"""Products of tensors in 8 bits by each kernel on purpose: tiles of 64, 128 and 256, the contraction whole and in parts, the kernel of up to 16 rows; sizes that no tile divides, seventeen and thirty-three
blocks, both formats on both sides, both result types.  That a shape takes the kernel it stands for is asserted: where the rule that chooses changes, the shapes here have to.

Tolerances: whole numbers have exact sums (compared bit for bit; bfloat16 the sum rounded once); others fp32 K 2^-24 of the sum of magnitudes, bfloat16 2^-10 of it and 2^-8 of the result."""
import ctypes as C

import pytest
import torch

from test_gpu_block8 import whole_numbers
from test_gpu_block8_ends import blocks

pytestmark = pytest.mark.gpu
F = torch.float64
FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
PAIRS = [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")]
# (m, n, k): tile and whether the contraction is in parts, for fp32 and bfloat16 results
CASES = [((13, 301, 2500), (0, False), (0, False)),
         ((131, 197, 515), (1, False), (1, False)),
         ((301, 499, 8190), (1, True), (1, True)),
         ((701, 5003, 900), (2, False), (2, False)),
         ((767, 769, 12605), (2, True), (2, True)),
         ((4001, 3897, 2050), (4, False), (4, False)),      # seventeen blocks, two places in the last
         ((3841, 4090, 4225), (4, False), (4, False)),      # thirty-four, one place in the last
         ((4095, 4095, 1930), (4, False), (4, False)),      # sixteen
         ((701, 3001, 12280), (4, True), (2, True)),
         ((1501, 2999, 6100), (1, False), (4, True))]
RUNS = [(size, t, cut) for size, f, b in CASES for t, cut in ((torch.float32, f), (torch.bfloat16, b))]


@pytest.fixture(scope="module")
def imu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2403_07339_amd import binding
    return binding


def test_every_kernel_is_among_them():
    for t in (torch.float32, torch.bfloat16):
        assert {cut for _, dtype, cut in RUNS if dtype == t} == {(0, False), (1, False), (1, True), (2, False), (2, True), (4, False), (4, True)}


def takes(imu, size, dtype, cut):
    tile, parts = imu.imunpack_diag_block8_cut(*size, dtype)
    assert (tile, parts > 1) == cut, (size, dtype, tile, parts)


@pytest.mark.parametrize("fa,fb", PAIRS)
@pytest.mark.parametrize("size,dtype,cut", RUNS)
def test_whole_numbers(imu, size, dtype, cut, fa, fb):
    takes(imu, size, dtype, cut)
    m, n, k = size
    a, b = whole_numbers(m, k, fa, m + n + k, 5), whole_numbers(n, k, fb, m * n + k, 5)
    want = a.cuda().double() @ b.cuda().double().t()
    qa, qb = imu.imunpack_block8_quantize(a.cuda(), fa)[0], imu.imunpack_block8_quantize(b.cuda(), fb)[0]
    assert torch.equal(imu.imunpack_block8_gemm(qa, qb, dtype), want.float().to(dtype))


@pytest.mark.parametrize("fa,fb", PAIRS)
@pytest.mark.parametrize("size,dtype,cut", RUNS)
def test_powers_of_two_of_every_block(imu, size, dtype, cut, fa, fb):
    """Random codes, a random power of two for each row and block; with a bias, into rows that are wider than the result, behind which nothing is written."""
    takes(imu, size, dtype, cut)
    m, n, k = size
    g = torch.Generator().manual_seed(m * 7 + n)
    kb = -(-k // 128)

    def operand(rows, fmt):
        x = torch.zeros(rows, kb * 128)
        x[:, :k] = torch.randn(rows, k, generator=g)
        codes, byte = x.to(FORMATS[fmt]), torch.randint(117, 135, (rows, kb), generator=g).to(torch.uint8)
        value = codes.to(F).cuda().view(rows, kb, 128).mul_(torch.exp2(byte.to(F).cuda() - 127)[:, :, None]).view(rows, -1)
        return blocks(imu, codes.view(torch.uint8), byte, fmt, behind=255), value

    (qa, va), (qb, vb) = operand(m, fa), operand(n, fb)
    bias = torch.randn(n, generator=g).cuda()
    want, size_of = va @ vb.t() + bias.to(F), va.abs_() @ vb.abs_().t() + bias.abs().to(F)
    limit = (k + 1) * 2.0 ** -24 * size_of if dtype == torch.float32 else 2.0 ** -10 * size_of + 2.0 ** -8 * want.abs()
    got = imu.imunpack_block8_gemm(qa, qb, dtype, bias=bias)
    assert ((got.to(F) - want).abs() <= limit).all()
    # the same through the C entry point, rows of the result `ldo` apart
    ldo, half = n + 21, int(dtype == torch.bfloat16)
    out = torch.full((m + 3, ldo), -7.0, dtype=dtype, device="cuda")
    bytes_ = C.c_size_t()
    f = imu._lib.imunpack_block8_gemm_workspace
    assert f(C.c_int64(m), C.c_int64(n), C.c_int64(k), C.c_int(half), C.byref(bytes_)) == 0 and (bytes_.value > 0) == cut[1]
    room = torch.full((bytes_.value + 64,), 77, dtype=torch.uint8, device="cuda")
    p, i64 = (lambda t: C.c_void_p(t.data_ptr())), C.c_int64
    code = {"e4m3": 0, "e5m2": 1}
    assert imu._lib.imunpack_block8_gemm(p(qa.codes), i64(kb * 128), p(qa.scales), i64(qa.scales.shape[1]), C.c_int(code[fa]), p(qb.codes), i64(kb * 128), p(qb.scales), i64(qb.scales.shape[1]),
                                         C.c_int(code[fb]), i64(m), i64(n), i64(k), p(bias), p(out), i64(ldo), C.c_int(half), p(room), bytes_, C.c_void_p(imu._stream())) == 0
    assert torch.equal(out[:m, :n], got)
    assert (out[m:] == -7).all() and (out[:, n:] == -7).all() and (room[bytes_.value:] == 77).all()
