"""The norms around a residual block: arguments the C interface refuses, with its
codes and messages, before any device work (no GPU needed), and the binding's
checks."""
import ctypes as C

import pytest
import torch

import paper_2609_16175_amd as boa
from paper_2609_16175_amd import ops

EINVAL = -1
P = 4096   # stands for a device pointer: refused calls never read it


def _call(grad, **over):
    a = ops.Block(dtype=1, param_dtype=1, rows=10, d=16, norm=0, post=1, pre=1, gate_rows=1, scale=1.0, eps=1e-5, x=P, x_stride=16,
                  f=P, f_stride=16, gate=P, gate_stride=16, post_weight=P, post_bias=P, weight=P, bias=P, h=P, y=P, stats=P, dh=P,
                  dh_stride=16, dy=P, dy_stride=16, dx=P, df=P, dgate=P, dpost_weight=P, dpost_bias=P, dweight=P, dbias=P,
                  workspace=P, workspace_bytes=1 << 40)
    for k, v in over.items():
        setattr(a, k, v)
    L = ops._lib()
    return (L.boa_block_norm_backward if grad else L.boa_block_norm)(C.byref(a), None)


def _err():
    return boa.lib().boa_last_error().decode()


@pytest.mark.parametrize("grad", [0, 1])
@pytest.mark.parametrize("over,needle", [
    (dict(dtype=3), "dtype"), (dict(param_dtype=2), "parameters"), (dict(norm=2), "norm"), (dict(rows=-1), "rows"),
    (dict(rows=1 << 31), "rows"), (dict(d=0), "d out of range"), (dict(d=(1 << 20) + 1), "d out of range"),
    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(scale=float("inf")), "scale"),
    (dict(scale=float("nan")), "scale"), (dict(x_stride=15), "stride"), (dict(f_stride=15), "stride"),
    (dict(gate_stride=15), "gate's row stride"), (dict(x=None), "NULL rows"), (dict(f=None), "NULL rows"),
])
def test_refuses(over, needle, grad):
    assert _call(grad, **over) == EINVAL and needle in _err()


@pytest.mark.parametrize("grad,over,needle", [
    (0, dict(h=None), "NULL output"), (0, dict(y=None), "NULL output"),
    (1, dict(dh_stride=15), "stride"), (1, dict(dy_stride=15), "stride"), (1, dict(dh=None, dy=None), "neither"),
    (1, dict(pre=0), "dy without"), (1, dict(stats=None), "stats"), (1, dict(gate=None), "without a gate"),
    (1, dict(post=0), "without it"), (1, dict(workspace=None), "workspace"), (1, dict(workspace=P + 8), "workspace"),
    (1, dict(workspace_bytes=64), "workspace"),
])
def test_refuses_one_way(grad, over, needle):
    assert _call(grad, **over) == EINVAL and needle in _err()


def test_nothing_to_do():
    assert _call(0, rows=0, x=None, f=None, h=None, y=None) == 0
    assert _call(1, dx=None, df=None, dgate=None, dpost_weight=None, dpost_bias=None, dweight=None, dbias=None, workspace=None) == 0
    assert ops._lib().boa_block_norm(None, None) == EINVAL and ops._lib().boa_block_norm_backward(None, None) == EINVAL


def test_workspace_is_bounded():
    ws = ops._lib().boa_block_norm_backward_workspace
    assert ws(8, 768) == (4 * 768 + 16) * 4 and ws(1 << 20, 1024) == (1024 * 4 * 1024 + (2 << 20)) * 4
    for d in (1, 4096, 16_384, 100_000, 1 << 20):
        for rows in (0, 1, 9, 1 << 13, (1 << 31) - 1):
            assert 0 < ws(rows, d) <= max(4 * d * 4, 1 << 27) + 8 * rows


def test_binding_refuses_host_tensors():
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError, match="device"):
        boa.block_norm(x, x)
    with pytest.raises(ValueError, match="device"):
        boa.block_norm_backward(x, x, x, x, torch.zeros(4, 2))
