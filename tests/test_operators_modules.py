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
