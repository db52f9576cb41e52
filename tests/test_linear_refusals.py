"""Linear layers: arguments the C interface refuses, with its codes and messages,
before any device work (no GPU needed), and the binding's checks."""
import ctypes as C

import pytest
import torch

import paper_2609_16175_amd as boa
from paper_2609_16175_amd import ops

EINVAL = -1
P = 4096   # stands for a device pointer: refused calls never read it


def _dense(**over):
    a = ops.Dense(dtype=1, activation=1, M=100, N=16, K=24, x=P, x_stride=24, w=P, w_stride=24, bias=P, param_dtype=1,
                  residual=P, residual_stride=16, y=P, pre=P, dy=P, dy_stride=16, dx=P, dw=P, dbias=P)
    for k, v in over.items():
        setattr(a, k, v)
    return a


def _call(grad, ws=P, n=1 << 40, **over):
    L = ops._lib()
    return (L.boa_linear_grad if grad else L.boa_linear)(C.byref(_dense(**over)), ws, n, None)


def _err():
    return boa.lib().boa_last_error().decode()


BOTH = [(dict(dtype=3), "dtype"), (dict(activation=5), "activation"), (dict(activation=-1), "activation"),
        (dict(M=-1), "M out of range"), (dict(M=1 << 31), "M out of range"), (dict(M=(1 << 31) - 255), "M out of range"), (dict(N=0), "N out of range"),
        (dict(N=(1 << 17) + 1), "N out of range"), (dict(K=0), "K out of range"), (dict(K=(1 << 17) + 1), "K out of range"),
        (dict(x_stride=23), "x's row stride"), (dict(w_stride=23), "w's row stride"), (dict(param_dtype=2), "bias"),
        (dict(x=None), "NULL x"), (dict(w=None), "NULL w")]


@pytest.mark.parametrize("grad", [0, 1])
@pytest.mark.parametrize("over,needle", BOTH)
def test_refuses(over, needle, grad):
    assert _call(grad, **over) == EINVAL and needle in _err()
    assert ops._lib().boa_linear_workspace(C.byref(_dense(**over)), grad) == EINVAL


@pytest.mark.parametrize("over,needle", [(dict(y=None), "NULL y"), (dict(residual_stride=15), "residual")])
def test_forward_refuses(over, needle):
    assert _call(0, **over) == EINVAL and needle in _err()


@pytest.mark.parametrize("over,needle", [(dict(dy=None), "NULL dy"), (dict(dy_stride=15), "dy's row stride"), (dict(pre=None), "NULL pre"),
                                         (dict(ws=None), "workspace"), (dict(ws=P + 8), "workspace"), (dict(n=64), "workspace")])
def test_backward_refuses(over, needle):
    assert _call(1, **over) == EINVAL and needle in _err()


def test_workspace():
    L = ops._lib()
    size = lambda grad, **over: L.boa_linear_workspace(C.byref(_dense(**over)), grad)  # noqa: E731
    assert size(0, M=64) == 0 and size(0, M=16, dtype=0, param_dtype=0) == 0
    # rows read in place take none, others a copy each; float32 rows two parts of 16 bits and the largest magnitudes
    assert size(0, M=8192, N=8192, K=8192, x_stride=8192, w_stride=8192, residual=None) == 0
    copy = 8192 * 8192 * 2
    assert size(0, M=8192, N=8192, K=8191, x_stride=8192, w_stride=8192, residual=None) == 2 * copy
    assert size(0, M=8192, N=8192, K=8192, x_stride=8192, w_stride=8192, residual=None, x=P + 2) == copy
    assert size(0, M=8192, N=8192, K=8192, x_stride=8192, w_stride=8192, residual=None, dtype=0, param_dtype=0) == 2 * (2 * copy + 8192 * 4)
    assert _call(0, M=129, dtype=0, param_dtype=0, n=16) == EINVAL and "workspace" in _err()
    assert L.boa_linear_workspace(None, 0) == EINVAL and L.boa_linear(None, P, 0, None) == EINVAL


def test_nothing_to_do():
    assert _call(0, M=0, x=None, y=None) == 0
    assert _call(1, dx=None, dw=None, dbias=None) == 0


def test_binding_refuses():
    x, w = torch.zeros(2, 8), torch.zeros(3, 8)
    with pytest.raises(ValueError, match="device"):
        boa.linear(x, w)
    with pytest.raises(ValueError, match="device"):
        boa.linear_backward(torch.zeros(2, 3), x, w)
