"""The layers, the norm, the loss and the optimiser together: a training step's gradients against autograd over plain operations on the same
activations, training that learns, and the integer head."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lm():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2403_07339_amd import lm
    return lm


def test_loss_end_of_the_model_against_plain_autograd(lm):
    """From the last block's outputs on (norm, head, loss) everything is fp32: 1e-5 of the gradients."""
    c = lm.Config(vocab=333, tokens=40, width=96, hidden=128, heads=3, layers=1)
    torch.manual_seed(3)
    model = lm.MaskedLM(c)
    tokens, target = lm.batch(c, 6, torch.Generator().manual_seed(4))
    x, stream = (t.detach().requires_grad_() for t in model.encode(tokens))
    loss = model.head(model.norm(x, stream)[0], target)
    loss.backward()
    f = torch.float64
    x6, s6, n6, w6 = (t.detach().to(f).requires_grad_() for t in (x, stream, model.norm.weight, model.head.weight))
    h = x6 + s6
    y = h / torch.sqrt((h * h).mean(-1, keepdim=True) + model.norm.eps) * n6
    want = torch.nn.functional.cross_entropy((y @ w6.t()).view(-1, c.vocab), target.view(-1), ignore_index=lm.IGNORE)
    want.backward()
    assert abs(float(loss.detach()) - float(want.detach())) < 1e-5
    for got, ref in ((x.grad, x6.grad), (stream.grad, s6.grad), (model.norm.weight.grad, n6.grad), (model.head.weight.grad, w6.grad)):
        assert float((got.to(f) - ref).norm() / ref.norm()) < 1e-5
    # the whole model: every parameter gets a finite gradient
    model(tokens, target).backward()
    for name, p in model.named_parameters():
        assert p.grad is not None and torch.isfinite(p.grad).all() and p.grad.any(), name


@pytest.mark.parametrize("bits", [32, 8])
def test_training_learns(lm, bits):
    """200 classes guessed at random cost log 200 = 5.3; in 200 steps the rule of the sequences brings a third of that (3.3 with states of
    either width), a quarter is asked for."""
    c = lm.Config(vocab=200, tokens=32, width=64, hidden=128, heads=2, layers=1, mask=0.2)
    model, losses = lm.train(c, 200, sequences=32, lr=5e-3, state_bits=bits)
    assert torch.isfinite(losses).all() and 4.5 < float(losses[0]) < 8.0
    assert float(losses[-20:].mean()) < 0.75 * 5.3


def test_integer_head(lm):
    """The logits of integers with steps: a row's are off by half a step of either operand through the product."""
    c = lm.Config(vocab=300, tokens=24, width=128, hidden=128, heads=2, layers=1)
    torch.manual_seed(5)
    model = lm.MaskedLM(c)
    with torch.no_grad():
        model.head.weight[::17, ::13] *= 30.0     # heavy hitters
        tokens, _ = lm.batch(c, 3, torch.Generator().manual_seed(6))
        x, stream = model.encode(tokens)
        head = lm.IntegerHead(model)
        y, _ = model.norm(x, stream)
        q, scale, h = model.norm.quantize(x, 8, stream)
        w, f = model.head.weight, torch.float64
        want = y.to(f) @ w.to(f).t()
        bound = (0.5 * scale.to(f)[..., None] * w.to(f).abs().sum(1) + 0.5 * head.step * y.to(f).abs().sum(-1, keepdim=True)
                 + 0.25 * c.width * scale.to(f)[..., None] * head.step) * 1.001
        for call in range(3):     # kept from the second call on, taken over by the third
            got = head(x, stream)
            assert head.plan.weights_reused() == (call == 2)
            assert ((got.to(f) - want).abs() <= bound).all()
            # and exactly the product of the integers, scaled
            exact = (q.to(f) @ head.Q.to(f).t()) * (scale.to(f)[..., None] * head.step)
            assert ((got.to(f) - exact).abs() <= 3 * 2.0 ** -24 * exact.abs()).all()


@pytest.mark.parametrize("bits,seed", [(8, 0), (32, 1), (32, 3)])
def test_training_goes_on(lm, bits, seed):
    """The model as it comes: attention that looks at few tokens leaves gradients of which all but a few entries are next to nothing, and no product may refuse them."""
    model, losses = lm.train(lm.Config(), 150, state_bits=bits, seed=seed)
    assert losses.numel() == 150 and torch.isfinite(losses).all()
    assert float(losses[-20:].mean()) < 0.8 * 6.9     # log 1000 at random
