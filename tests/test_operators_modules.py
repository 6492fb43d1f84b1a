"""What the modules around the products ask of the binding, with the binding's functions replaced by ones that write down their arguments (no GPU)."""
import pytest
import torch


@pytest.fixture(scope="module")
def imu():
    from paper_2403_07339_amd import build
    import os
    if not os.path.exists(build.LIB):
        build.build()
    from paper_2403_07339_amd import binding
    return binding


@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
def test_loss_makes_gradients_only_where_they_may_be_asked_for(imu, monkeypatch, reduction):
    from paper_2403_07339_amd import loss
    asked = []

    def xent(x, w, target, ignore_index=-100, reduction="mean", want_grad=False, want_x=True, want_w=True):
        asked.append((want_grad, want_x, want_w))
        return torch.zeros(target.shape if reduction == "none" else ()), imu.XentSaved(ignore_index, reduction) if want_grad else None

    monkeypatch.setattr(imu, "imunpack_xent", xent)
    head = loss.LinearCrossEntropy(8, 20, reduction=reduction)
    x, target = torch.randn(5, 8), torch.randint(0, 20, (5,))
    with torch.no_grad():
        assert not head(x, target).requires_grad
        head(x.clone().requires_grad_(), target)
    with torch.inference_mode():
        head(x, target)
    loss.linear_cross_entropy(x, head.weight.detach(), target, reduction=reduction)
    assert [a[0] for a in asked] == [False] * 4
    assert head(x, target).requires_grad and asked[-1] == (True, False, True)
    loss.linear_cross_entropy(x.clone().requires_grad_(), head.weight.detach(), target, reduction=reduction)
    assert asked[-1] == (True, True, False)


@pytest.fixture
def adamw_calls(imu, monkeypatch):
    """optim.AdamW on the CPU: the step's formulas in torch, and what each call of the binding was given."""
    calls = []

    def adamw(params, grads, exp_avg, exp_avg_sq, step, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, m_scales=None, v_scales=None, copies=None, seed=0):
        calls.append(dict(params=params, grads=grads, step=step, seed=seed & 0xFFFFFFFF, copies=copies))
        for k, (p, g, m, v) in enumerate(zip(params, grads, exp_avg, exp_avg_sq)):
            if g.dtype not in (torch.float32, torch.bfloat16) or not all(t.is_contiguous() for t in (p, g, m, v)):
                raise ValueError("adamw: a tensor of the wrong type or layout")
            if m_scales is None:
                m.lerp_(g.float(), 1 - beta1)
                v.lerp_(g.float() ** 2, 1 - beta2)
                p.mul_(1 - lr * weight_decay).addcdiv_(m, (v / (1 - beta2 ** step)).sqrt() + eps, value=-lr / (1 - beta1 ** step))
                if copies is not None:
                    copies[k].data.copy_(p)

    monkeypatch.setattr(imu, "imunpack_adamw", adamw)
    return calls


@pytest.mark.parametrize("bits", [32, 8])
def test_states_of_the_other_width_are_refused(adamw_calls, bits):
    from paper_2403_07339_amd import optim
    def make(bits):
        p = torch.nn.Parameter(torch.ones(512))   # (as many codes as elements)
        p.grad = torch.ones(512)
        o = optim.AdamW([p], state_bits=bits)
        o.step()
        return o
    mine, other = make(bits), make(40 - bits)
    with pytest.raises(ValueError):
        mine.load_state_dict(other.state_dict())
    mine.load_state_dict(make(bits).state_dict())
    optim.AdamW([torch.nn.Parameter(torch.ones(512))], state_bits=bits).load_state_dict(mine.state_dict())


def test_a_step_is_seen_by_autograd(adamw_calls):
    """A graph that saved a parameter before the step must not go backward with the new values."""
    from paper_2403_07339_amd import optim
    p, copy = torch.nn.Parameter(torch.ones(4)), torch.ones(4, dtype=torch.bfloat16)
    idle = torch.nn.Parameter(torch.ones(4))
    y = (p * p).sum() + (idle * idle).sum()
    p.grad = torch.ones(4)
    before = copy._version
    optim.AdamW([p, idle], copies={p: copy}).step()
    assert copy._version > before and idle._version == 0
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_calls_of_one_step_round_with_their_own_random_bits(adamw_calls):
    """Gradients of two types, or some parameters with copies, go in calls of their own, each of which numbers its tensors from 0."""
    from paper_2403_07339_amd import optim
    ps = [torch.nn.Parameter(torch.ones(4)) for _ in range(6)]
    o = optim.AdamW([dict(params=ps[:3]), dict(params=ps[3:])], state_bits=8, seed=5, copies={p: torch.ones(4, dtype=torch.bfloat16) for p in (ps[1], ps[2], ps[4])})
    for _ in range(2):
        for p in ps:
            p.grad = torch.ones(4)
        o.step()
    assert len(adamw_calls) == 8 and adamw_calls[0]["seed"] == 5
    assert len({c["seed"] for c in adamw_calls[:4]}) == 4
    # the kernel's key of a call is made of seed + step * 0x9E3779B1: no two calls of a few thousand steps meet there
    seeds = [c["seed"] for c in adamw_calls[:4]]
    keys = {(s + t * 0x9E3779B1) & 0xFFFFFFFF for s in seeds for t in range(1, 5001)}
    assert len(keys) == 4 * 5000
    again = optim.AdamW([dict(params=ps[:3]), dict(params=ps[3:])], state_bits=8, seed=5, copies=o.copies)
    again.step()
    assert [c["seed"] for c in adamw_calls[8:]] == seeds


def test_a_refused_step_is_none(adamw_calls):
    from paper_2403_07339_amd import optim
    p = torch.nn.Parameter(torch.ones(4, dtype=torch.float64))
    o = optim.AdamW([p])
    p.grad = torch.ones(4, dtype=torch.float64)
    with pytest.raises(ValueError):
        o.step()
    assert o.state[p]["step"] == 0


def test_a_step_is_not_captured(adamw_calls, monkeypatch):
    """The step's number and its random bits are arguments: a graph would repeat those of the captured step."""
    from paper_2403_07339_amd import optim
    monkeypatch.setattr(optim, "_capturing", lambda: True)
    p = torch.nn.Parameter(torch.ones(4))
    p.grad = torch.ones(4)
    o = optim.AdamW([p])
    with pytest.raises(RuntimeError, match="captured"):
        o.step()
    assert not adamw_calls and not o.state


@pytest.mark.parametrize("bits", [32, 8])
def test_parameters_of_any_layout(adamw_calls, bits):
    """Transposed, strided and channels-last parameters step as their contiguous copies do."""
    from paper_2403_07339_amd import optim
    torch.manual_seed(1)
    start = [torch.randn(6, 5).t(), torch.randn(8, 6)[:, ::2], torch.randn(2, 3, 4, 4).contiguous(memory_format=torch.channels_last), torch.randn(7)]
    mine = [torch.nn.Parameter(t) for t in start]
    want = [torch.nn.Parameter(t.detach().clone(memory_format=torch.contiguous_format)) for t in start]
    assert [p.is_contiguous() for p in mine] == [False, False, False, True]
    a, b = optim.AdamW(mine, state_bits=bits, lr=0.1), optim.AdamW(want, state_bits=bits, lr=0.1)
    for k in range(3):
        for p, q in zip(mine, want):
            q.grad = torch.randn(q.shape)
            p.grad = q.grad.clone()
        if k == 2:
            again = optim.AdamW(mine, state_bits=bits, lr=0.1)
            again.load_state_dict(a.state_dict())
            a = again
        a.step()
        b.step()
    for p, q in zip(mine, want):
        assert torch.equal(p, q) and p.stride() == start[mine_index(mine, p)].stride()


def mine_index(some, one):
    return next(k for k, p in enumerate(some) if p is one)


def refused_on_other_devices(imu, one, other):
    """Calls with a tensor of another device than the rest are refused, before anything is read or launched (fake tensors have no memory)."""
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        def at(device, *shape, dtype=torch.float32):
            return torch.empty(shape, device=device, dtype=dtype)
        x, w, rstd = (lambda d: at(d, 4, 8)), (lambda d: at(d, 8)), (lambda d: at(d, 4))
        target = lambda d: at(d, 4, dtype=torch.int64)  # noqa: E731
        scalar, head = (lambda d: at(d)), (lambda d: at(d, 20, 8))
        xent = imu.XentSaved
        for make, call in (
                ((x, w, x), lambda a, b, c: imu.imunpack_rmsnorm(a, b, residual=c)),
                ((x, w, x), lambda a, b, c: imu.imunpack_rmsnorm_quantize(a, b, residual=c)),
                ((x, x, w, rstd, x), lambda g, h, w, r, gh: imu.imunpack_rmsnorm_backward(g, h, w, imu.NormSaved(r), gh)),
                ((x, head, target), lambda a, b, t: imu.imunpack_xent(a, b, t)),
                ((x, head, target, scalar), lambda a, b, t, g: imu.imunpack_xent_backward(a, b, t, xent(-100, "mean"), g)),
                ((x, head, target, scalar, x, head), lambda a, b, t, g, gx, gw: imu.imunpack_xent_backward(a, b, t, xent(-100, "mean", gx, gw), g)),
                ((w, w, w, w), lambda p, g, m, v: imu.imunpack_adamw([p], [g], [m], [v], step=1))):
            for k in range(len(make)):
                with pytest.raises(ValueError):
                    call(*[f(other if i == k else one) for i, f in enumerate(make)])


def test_tensors_of_several_devices_are_refused(imu, monkeypatch):
    monkeypatch.setattr(imu, "_stream", lambda: 0)
    refused_on_other_devices(imu, "cuda:0", "cuda:1")


@pytest.mark.gpu
def test_tensors_of_another_device_than_the_current_are_refused(imu):
    if torch.cuda.device_count() < 2:
        pytest.skip("needs two devices")
    x, w = torch.zeros(4, 8, device="cuda:1"), torch.zeros(8, device="cuda:1")
    with torch.cuda.device(0):
        for call in (lambda: imu.imunpack_rmsnorm(x, w), lambda: imu.imunpack_rmsnorm_quantize(x, w), lambda: imu.imunpack_adamw([w], [w], [w], [w], step=1),
                     lambda: imu.imunpack_xent(x, torch.zeros(20, 8, device="cuda:1"), torch.zeros(4, dtype=torch.int64, device="cuda:1"))):
            with pytest.raises(ValueError):
                call()
