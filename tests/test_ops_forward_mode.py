"""Operators with an autograd form refuse forward-mode tangents, which they do
not carry on, in place of dropping them (no GPU needed: the library's calls are
replaced)."""
import pytest
import torch
from torch.autograd import forward_ad

import paper_2609_16175_amd as boa
from paper_2609_16175_amd import ops


@pytest.fixture
def plain(monkeypatch):
    def linear_forward(x, weight, bias=None, residual=None, activation="none", keep=False, stream=None):
        y = x @ weight.t()
        return y if bias is None else y + bias, None

    def xent(name, h, rows, labels, bias, scale, reduction, stream, grad, *rest):
        z = torch.zeros(())
        return ops.XentResult(z, z, *(z,) * 3 if grad else ())

    monkeypatch.setattr(ops, "linear_forward", linear_forward)
    monkeypatch.setattr(ops, "_xent", xent)


def tensors():
    return [torch.ones(2, 3), torch.ones(4, 3), torch.ones(4), torch.ones(2, 4)]


@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("which", range(4))
def test_linear(plain, which, grad):
    t = tensors()
    with forward_ad.dual_level(), torch.set_grad_enabled(grad):
        t[which] = forward_ad.make_dual(t[which], torch.ones_like(t[which]))
        with pytest.raises(NotImplementedError, match="forward mode"):
            boa.linear(*t)


@pytest.mark.parametrize("which", [0, 1, 3])
def test_softmax_xent(plain, which):
    t = [torch.ones(2, 3), torch.ones(4, 3), torch.zeros(2, dtype=torch.int64), torch.ones(4)]
    with forward_ad.dual_level():
        t[which] = forward_ad.make_dual(t[which], torch.ones_like(t[which]))
        for reduction in ("mean", "none"):
            with pytest.raises(NotImplementedError, match="forward mode"):
                boa.softmax_xent(*t, reduction=reduction)


def test_without_tangents(plain):
    t = tensors()
    want = t[0] @ t[1].t() + t[2]
    with forward_ad.dual_level():
        assert torch.equal(boa.linear(*t), want)
    assert torch.equal(boa.linear(*t), want) and not boa.linear(*t).requires_grad
    t[1].requires_grad_()
    assert boa.linear(*t).requires_grad
