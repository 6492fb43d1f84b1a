"""GELU and SiLU of negative inputs, whose values are a small part of the inputs: against the definitions in binary64, relative to the value itself.

Tolerances, in units of 2^-24 of the value.  GELU is u phi(u) R(u): phi's exponent u^2 / 2 is off by 1.5 of itself (its square and the product with a constant of 24 bits), 0.75 u^2 in phi; exp2 2, its factor
1.5, R 8, three products 3: below 16 + u^2.  SiLU is u / (1 + exp(-u)): exp 4 (twice the error of its own), the sum, the quotient: below 16.  Slopes are differences of such numbers, Phi and u phi (sig and
sig u (1 - sig)), each within 16 + u^2 of its own size; nothing counts below 2^-120 (phi is 0 where binary32's normal numbers end)."""
import pytest
import torch

from test_gpu_block8 import check_codes, definition, exponents

pytestmark = pytest.mark.gpu
F = torch.float64


@pytest.fixture(scope="module")
def imu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2403_07339_amd import binding
    return binding


def below64(u):
    return torch.special.erfc(u * -0.7071067811865476) / 2   # (torch.special.ndtr is 0 from -8.4 on: it is taken as (1 + erf) / 2)


def act64(u, act):
    return u * below64(u) if act == "gelu" else u * torch.sigmoid(u)


def parts64(u, act):
    """The two terms of the slope."""
    if act == "gelu":
        return below64(u), u * torch.exp(-u * u / 2) * 0.3989422804014327
    sig = torch.sigmoid(u)
    return sig, u * sig * torch.sigmoid(-u)


def units(u, act):
    return (16 + (u * u if act == "gelu" else 0 * u)) * 2.0 ** -24


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_values_and_slopes(imu, dtype, act):
    u = torch.cat([torch.linspace(-13, 13, 100001), -torch.logspace(-30, 0, 2001), torch.logspace(-30, 0, 2001), torch.zeros(1)]).to(dtype).cuda()
    y, _, kept = imu.imunpack_act8(u, act)
    want = act64(u.to(F), act)
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    assert ((y.to(F) - want).abs() <= (units(u.to(F), act) + step) * want.abs() + 2.0 ** -120).all()
    v = kept[0].values().to(F)[0]
    gu = imu.imunpack_act8_backward(torch.ones_like(u), kept, act).to(F)
    one, two = parts64(v, act)
    assert ((gu - one - two).abs() <= units(v, act) * (one.abs() + two.abs()) + step * (one + two).abs() + 2.0 ** -120).all()


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_blocks_of_negative_inputs_alone(imu, dtype, gated, act):
    """Results in 8 bits of blocks whose inputs are all negative: the power of two is that of the largest result, and no value is further off than the format's own rounding."""
    g = torch.Generator().manual_seed(5)
    low = -torch.arange(1, 27).float()[:, None] / 2 - torch.rand(26, 384, generator=g)
    u = (torch.cat([low, torch.randn(26, 384, generator=g)], 1) if gated else low).to(dtype).cuda()
    parts = list(u.to(F).split(384, 1))
    want = act64(parts[0], act) * (parts[1] if gated else 1.0)
    rel = units(parts[0], act) + 2.0 ** -23
    y, codes, kept = imu.imunpack_act8(u, act, gated, quantize=True)
    scale = torch.exp2(exponents(codes)).cuda()
    wide = scale.repeat_interleave(128, 1)
    v = codes.values().to(F)
    assert ((v - want).abs() <= (2.0 ** -4 + rel) * want.abs() + 2.0 ** -10 * wide + 2.0 ** -120).all()
    top = want.abs().reshape(26, 3, 128).amax(2)
    worst = rel.reshape(26, 3, 128).amax(2)
    counted = top > 2.0 ** -100   # (what lies below 2^-120 may be anything up to that, a millionth of the largest here)
    assert ((top <= 448.0 * scale * (1 + worst)) | ~counted).all() and ((top * (1 + worst) > 224.0 * scale) | ~counted).all() and float(counted.to(F).mean()) > 0.8
    assert torch.equal(y.to(F), v.to(dtype).to(F))
    for part, k in zip(parts, kept):
        check_codes(k, *definition(part, "e4m3"), "e4m3", 384)


def test_what_eight_bits_leave_of_slopes_and_factors(imu):
    """Inputs of a normal distribution.  A value of 8 bits is off by up to half a step, 2^-4 of the power of two below it, evenly: in the mean 2^-5 of that, which is 2^-5 times the mean of 1 / m over fractions m in
    [1, 2), 0.69 (m even) to 0.72 (its logarithm even), of the value: 0.022.  A slope moves by that error times f'', at most 0.8 (GELU at 0; 0.5 SiLU): its root mean square, of e = rms 0.027 |u| where f'' is large, stays
    below 0.8 * 0.027 * 0.5 = 0.011 of slopes of about 1."""
    g = torch.Generator().manual_seed(0)
    u = torch.randn(512, 4096, generator=g).cuda()
    ones = torch.ones_like(u)
    for act in ("gelu", "silu"):
        _, _, kept = imu.imunpack_act8(u, act)
        off = (kept[0].values().to(F) - u.to(F)).abs() / u.to(F).abs()
        assert 0.0215 < float(off.mean()) < 0.0235
        slope = sum(parts64(u.to(F), act))
        gu = imu.imunpack_act8_backward(ones, kept, act).to(F)
        assert 0.007 < float((gu - slope).norm() / slope.norm()) < 0.011
