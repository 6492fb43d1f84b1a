"""The linear layer and the MLP in 8-bit floating point, log probabilities as an autograd function, and the model that runs them: against the definitions in
binary64 with the same 8-bit values, and for what is kept between the passes.

Tolerances.  The operands' values are equal bit for bit where x, the weights or the gradient are given (tests of the binding hold that), so a layer's results are off by the sums alone:
2e-6 of the norm in fp32 (sums of binary32), 2^-8 in bfloat16.  Behind an activation function an element next to the border between two codes may go the other way, 2^-3 of itself: with 2^-19 of an
element's error (16 * 2^-24, taken twice) and a border for every 2^-4 of its size, fewer than one in 2^14 does, which moves a product's result by less than 2^-3 / 2^7 = 2^-10 of its norm."""
import pytest
import torch

from test_gpu_block8 import act64, definition

pytestmark = pytest.mark.gpu
F = torch.float64


@pytest.fixture(scope="module")
def b8():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2403_07339_amd import block8
    return block8


def near(got, want, dtype, more=0.0):
    want = want.detach().to(got.device)
    limit = (2.0 ** -8 if dtype == torch.bfloat16 else 2e-6) + more
    assert got.dtype == dtype and got.shape == want.shape
    assert float((got.to(F) - want).norm()) <= limit * float(want.norm()) + 1e-30


def value(x, square=False):
    return definition(x.detach().reshape(-1, x.shape[-1]), "e4m3", square)[0].cuda()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lead,d,out", [((1,), 64, 64), ((3, 5), 100, 37), ((197,), 256, 1000), ((2, 300), 768, 130)])
def test_linear(b8, lead, d, out, dtype):
    torch.manual_seed(d + out)
    layer = b8.Block8Linear(d, out, device="cuda", dtype=dtype)
    x = (torch.randn(*lead, d, device="cuda") * 3).to(dtype).requires_grad_()
    gy = (torch.randn(*lead, out, device="cuda") * 1e-3).to(dtype)
    y = layer(x)
    y.backward(gy)
    g = gy.reshape(-1, out)
    vx, vw = value(x), value(layer.weight, True)
    near(y.detach().reshape(-1, out), vx @ vw.t() + layer.bias.to(F), dtype)
    near(x.grad.reshape(-1, d), value(g) @ vw, dtype)
    near(layer.weight.grad, definition(g.t(), "e4m3")[0].cuda() @ definition(vx.t(), "e4m3")[0].cuda().t(), dtype)
    near(layer.bias.grad, g.to(F).sum(0), dtype)
    frozen = layer.frozen()
    assert torch.equal(frozen(x), y.detach())
    with torch.no_grad():
        assert torch.equal(layer(x), y.detach())


def test_activations_and_parameters_of_different_types(b8):
    torch.manual_seed(1)
    layer = b8.Block8Linear(130, 70, device="cuda")
    x = torch.randn(40, 130, device="cuda").bfloat16().requires_grad_()
    gy = torch.randn(40, 70, device="cuda").bfloat16()
    y = layer(x)
    y.backward(gy)
    vx, vw = value(x), value(layer.weight, True)
    near(y.detach(), vx @ vw.t() + layer.bias.to(F), torch.bfloat16)
    near(x.grad, value(gy) @ vw, torch.bfloat16)
    near(layer.weight.grad, value(gy.t()) @ value(vx.t().cpu()).t(), torch.float32)
    near(layer.bias.grad, gy.to(F).sum(0), torch.float32)


def test_what_is_kept_between_the_passes(b8):
    layer = b8.Block8MLP(256, 512, act="silu", gated=True, device="cuda")
    x = torch.randn(1024, 256, device="cuda", requires_grad=True)
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t) or t, lambda t: t):
        y = layer(x)
    rows, room = 1024, 1024 * 16   # (a row's powers of two are filled up to 16 bytes)
    assert all(t.element_size() == 1 for t in kept)
    activations = sum(t.numel() for t in kept if t.shape[0] == rows and t.dtype == torch.float8_e4m3fn)
    assert activations == rows * (256 + 512 + 2 * 512)     # x, the result of the activation function, both halves of its input
    assert sum(t.numel() for t in kept if t.dtype == torch.float8_e8m0fnu and t.shape[0] == rows) == 4 * room
    y.sum().backward()
    kept.clear()
    with torch.no_grad(), torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t) or t, lambda t: t):
        layer(x)
    assert not kept


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("act,gated", [("gelu", False), ("silu", True), ("gelu", True)])
@pytest.mark.parametrize("rows,d,hidden", [(5, 64, 128), (300, 200, 333), (256, 384, 1000)])
def test_mlp(b8, rows, d, hidden, act, gated, dtype):
    """Step by step with the 8-bit values that the library made: each product and each slope against binary64."""
    from paper_2403_07339_amd import binding as imu
    torch.manual_seed(rows + hidden)
    layer = b8.Block8MLP(d, hidden, act, gated, device="cuda", dtype=dtype)
    x = torch.randn(rows, d, device="cuda").mul(2).to(dtype).requires_grad_()
    gy = torch.randn(rows, d, device="cuda").mul(1e-2).to(dtype)
    y = layer(x)
    y.backward(gy)
    w1, w2 = value(layer.up.weight, True), value(layer.down.weight, True)
    b1, b2 = layer.up.bias.detach().to(F), layer.down.bias.detach().to(F)
    u = (value(x) @ w1.t() + b1).to(dtype)
    parts = list(u.to(F).split(hidden, 1))
    a = act64(parts[0], act) * (parts[1] if gated else 1.0)
    more = 2.0 ** -9 if dtype == torch.float32 else 2.0 ** -6   # (bfloat16: u itself is rounded one way or the other beforehand, 2^-8 of it, and more codes with it)
    near(y.detach(), value(a.cpu()).to(F) @ w2.t() + b2, dtype, more)
    kept = [value(p.cpu()).requires_grad_() for p in parts]
    (act64(kept[0], act) * (kept[1] if gated else 1.0)).backward(value(gy) @ w2)
    gu = torch.cat([k.grad for k in kept], 1)
    near(x.grad, value(gu.cpu()) @ w1, dtype, more)
    near(layer.down.weight.grad, value(gy.t()) @ value(value(a.cpu()).t().cpu()).t(), dtype, more)
    near(layer.up.weight.grad, value(gu.t().cpu()) @ value(value(x).t().cpu()).t(), dtype, more)
    near(layer.up.bias.grad, gu.sum(0), dtype, more)
    near(layer.down.bias.grad, gy.to(F).sum(0), dtype)
    # the same as the binding's calls one after the other
    q, _ = imu.imunpack_block8_quantize(x.detach())
    h = imu.imunpack_block8_gemm(q, imu.imunpack_block8_quantize(layer.up.weight.detach(), square=True)[0], dtype, layer.up.bias.detach().float())
    _, codes, _ = imu.imunpack_act8(h, act, gated, quantize=True, keep=False, want_y=False)
    again = imu.imunpack_block8_gemm(codes, imu.imunpack_block8_quantize(layer.down.weight.detach(), square=True)[0], dtype, layer.down.bias.detach().float())
    assert torch.equal(again, y.detach())


def test_gradients_where_only_some_are_asked_for(b8):
    torch.manual_seed(2)
    layer = b8.Block8MLP(96, 160, "gelu", False, device="cuda")
    x, gy = torch.randn(70, 96, device="cuda"), torch.randn(70, 96, device="cuda")
    full = x.clone().requires_grad_()
    layer(full).backward(gy)
    want = {n: p.grad.clone() for n, p in layer.named_parameters()}
    for names in (["up.weight"], ["down.weight"], ["up.bias"], ["down.bias"], ["up.weight", "down.bias"], []):
        for n, p in layer.named_parameters():
            p.grad = None
            p.requires_grad_(n in names)
        v = x.clone().requires_grad_(not names)
        layer(v).backward(gy)
        for n, p in layer.named_parameters():
            assert (p.grad is None) == (n not in names) and (n not in names or torch.equal(p.grad, want[n]))
        assert bool(names) or torch.equal(v.grad, full.grad)


def test_empty_and_expanded_and_refused(b8):
    layer, mlp = b8.Block8Linear(64, 32, device="cuda"), b8.Block8MLP(64, 96, "silu", True, device="cuda")
    for module, out in ((layer, 32), (mlp, 64)):
        x = torch.zeros(0, 7, 64, device="cuda", requires_grad=True)
        y = module(x)
        assert y.shape == (0, 7, out)
        y.sum().backward()
        assert x.grad.shape == x.shape and all(not p.grad.any() for p in module.parameters())
        z = torch.randn(9, 64, device="cuda", requires_grad=True)
        module(z).sum().backward()       # (the gradient of a sum is one number, expanded)
        assert z.grad.any()
        row = torch.randn(64, device="cuda", requires_grad=True)
        assert module(row).shape == (out,)
        module(row.expand(5, 64)).sum().backward()
        assert row.grad.shape == (64,)
        with pytest.raises(ValueError):
            module(torch.randn(3, 65, device="cuda"))
        with pytest.raises(ValueError):
            module(torch.randn(3, 64, device="cuda").half())
    with pytest.raises(ValueError):
        b8.block8_mlp(z, mlp.up.weight, mlp.down.weight, act="silu", gated=False)
    with pytest.raises(ValueError):
        b8.block8_mlp(z, mlp.up.weight, mlp.down.weight, act="relu", gated=True)


def test_log_probs_as_a_function(b8):
    from paper_2403_07339_amd.logprobs import log_probs
    torch.manual_seed(4)
    x = torch.randn(3, 11, 500, device="cuda", requires_grad=True)
    t = torch.randint(0, 500, (3, 11), device="cuda")
    t[1, 4] = -100
    got = log_probs(x, t, top=3)
    assert got.logp.shape == (3, 11) and got.top_logp.shape == (3, 11, 3) and not got.top_index.requires_grad
    c = torch.randn(3, device="cuda")
    (c[0] * got.logp.sum() + c[1] * got.entropy.sum() + c[2] * got.top_logp.sum()).backward()
    z = x.detach().to(F).requires_grad_()
    logp = torch.log_softmax(z, -1)
    picked = torch.where(t >= 0, logp.gather(-1, t.clamp_min(0)[..., None])[..., 0], 0.0)
    (c[0] * picked.sum() - c[1] * (logp.exp() * logp).sum() + c[2] * logp.gather(-1, got.top_index).sum()).backward()
    assert float((x.grad - z.grad).abs().max()) < 1e-5 and float((got.logp - picked).abs().max()) < 1e-5
    first = x.grad.clone()
    x.grad = None
    log_probs(x, None).entropy.sum().backward()
    assert x.grad.any() and not torch.equal(x.grad, first)
    assert not log_probs(x.detach(), t).logp.requires_grad


def test_model_with_an_mlp_in_8_bits(b8):
    from paper_2403_07339_amd import lm
    c = lm.Config(vocab=200, tokens=32, width=64, hidden=128, heads=2, layers=2, mask=0.2, mlp="block8")
    torch.manual_seed(7)
    model = lm.MaskedLM(c)
    tokens, target = lm.batch(c, 8, torch.Generator().manual_seed(8))
    model(tokens, target).backward()
    for name, p in model.named_parameters():
        assert p.grad is not None and torch.isfinite(p.grad).all() and p.grad.any(), name
    trained, losses = lm.train(c, 30, sequences=16)
    assert losses.numel() == 30 and torch.isfinite(losses).all()
    got = lm.score(trained, lm.IntegerHead(trained), tokens, target)
    at = target != lm.IGNORE
    assert not got.logp[~at].any() and (got.logp[at] < 0).all() and (got.entropy > 0).all() and got.top_index.shape == (*tokens.shape, 5)
    assert (got.top_logp[..., :-1] >= got.top_logp[..., 1:]).all()
    with pytest.raises(ValueError):
        lm.MaskedLM(lm.Config(mlp="float"))
