"""A linear layer with weights in 8 bits alone: gradients of its input.

Tolerances: the operands' values are equal bit for bit, so that a gradient is off by its sums alone: 2e-6 of the norm in fp32, 2^-8 in bfloat16 (as for the layer that trains)."""
import pytest
import torch

from test_gpu_block8_modules import near, value

pytestmark = pytest.mark.gpu
F = torch.float64


@pytest.fixture(scope="module")
def b8():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2403_07339_amd import block8
    return block8


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lead,d,out", [((1,), 64, 64), ((), 130, 20), ((3, 5), 100, 37), ((2, 300), 768, 130)])
def test_gradient_of_the_input(b8, lead, d, out, dtype):
    torch.manual_seed(d + out)
    layer = b8.Block8Linear(d, out, device="cuda", dtype=dtype)
    frozen = layer.frozen()
    x = (torch.randn(*lead, d, device="cuda") * 3).to(dtype).requires_grad_()
    gy = (torch.randn(*lead, out, device="cuda") * 1e-3).to(dtype)
    y = frozen(x)
    assert y.requires_grad and torch.equal(y, layer(x))
    y.backward(gy)
    near(x.grad.reshape(-1, d), value(gy) @ value(layer.weight, True), dtype)
    assert layer.weight.grad is None and layer.bias.grad is None
    with torch.no_grad():
        assert not frozen(x).requires_grad and torch.equal(frozen(x), y)
    assert not frozen(x.detach()).requires_grad


def test_parameters_in_front_of_it_train(b8):
    """What stands before a frozen layer gets the gradient that it gets before one that trains."""
    torch.manual_seed(3)
    layer = b8.Block8Linear(96, 40, device="cuda")
    frozen = layer.frozen()
    first = torch.nn.Linear(50, 96, device="cuda")
    x, gy = torch.randn(70, 50, device="cuda"), torch.randn(70, 40, device="cuda")
    got = torch.autograd.grad(frozen(first(x)), list(first.parameters()), gy)
    want = torch.autograd.grad(layer(first(x)), list(first.parameters()), gy)
    assert all(float((a - b).norm()) <= 4e-6 * float(b.norm()) for a, b in zip(got, want))
    gy1 = torch.ones((), device="cuda")
    g = torch.autograd.grad(frozen(first(x)).sum(), first.weight, gy1)[0]     # (a gradient of stride 0)
    w = torch.autograd.grad(layer(first(x)).sum(), first.weight, gy1)[0]
    assert float((g - w).norm()) <= 4e-6 * float(w.norm())
    empty = torch.zeros(0, 96, device="cuda", requires_grad=True)
    frozen(empty).sum().backward()
    assert empty.grad.shape == (0, 96)
    with pytest.raises(ValueError):
        frozen(torch.zeros(3, 95, device="cuda", requires_grad=True))
