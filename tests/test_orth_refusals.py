"""Orthogonalised updates: arguments the C interface refuses, with its codes and
messages, before any device work (no GPU needed)."""
import ctypes as C

import pytest
import torch

import paper_2609_16175_amd as boa
from paper_2609_16175_amd import ops

EINVAL = -1
P = 4096   # stands for a device pointer: refused calls never read it
CO = (C.c_float * 96)(*([3.4445, -4.775, 2.0315] * 32))


def _orth(**over):
    a = ops.Orth(dtype=1, rows=20, cols=30, count=2, update=P, update_stride=30, update_batch=600, steps=5,
                 coefficients=C.addressof(CO), eps=1e-7, out=P)
    for k, v in over.items():
        setattr(a, k, v)
    return a


def _err():
    return boa.lib().boa_last_error().decode()


@pytest.mark.parametrize("over,needle", [
    (dict(dtype=4), "dtype"), (dict(count=-1), "count"), (dict(count=65536), "count"), (dict(rows=0), "rows and cols"),
    (dict(cols=0), "rows and cols"), (dict(rows=(1 << 14) + 1), "rows and cols"), (dict(cols=(1 << 14) + 1), "rows and cols"),
    (dict(steps=0), "steps"), (dict(steps=33), "steps"), (dict(coefficients=None), "coefficients"), (dict(eps=-1.0), "eps"),
    (dict(eps=float("nan")), "eps"), (dict(update_stride=29), "stride"), (dict(update=None), "NULL"), (dict(out=None), "NULL"),
])
def test_refuses(over, needle):
    a = _orth(**over)
    assert ops._lib().boa_orthogonalize(C.byref(a), P, 1 << 40, None) == EINVAL and needle in _err()
    assert ops._lib().boa_orthogonalize_workspace(C.byref(a)) == EINVAL


def test_refuses_coefficients_that_are_not_finite():
    bad = (C.c_float * 15)(*([1.0] * 14 + [float("inf")]))
    a = _orth(coefficients=C.addressof(bad))
    assert ops._lib().boa_orthogonalize(C.byref(a), P, 1 << 40, None) == EINVAL and "finite" in _err()


def test_workspace():
    L = ops._lib()
    need = L.boa_orthogonalize_workspace(C.byref(_orth(rows=1024, cols=4096, count=1, update_stride=4096)))
    # X in float32 and twice in f16, A and b A + c A^2 in f16
    assert need >= 1024 * 4096 * 8 + 1024 * 1024 * 4 and need < 1024 * 4096 * 8 + 1024 * 1024 * 4 + 4096
    for ws, n in ((None, 1 << 40), (P + 8, 1 << 40), (P, 64)):
        assert L.boa_orthogonalize(C.byref(_orth(rows=100, cols=90, update_stride=90)), ws, n, None) == EINVAL and "workspace" in _err()
    assert L.boa_orthogonalize_workspace(C.byref(_orth())) == 0   # 20 x 30: in one block
    assert L.boa_orthogonalize(C.byref(_orth(count=0, update=None, out=None)), None, 0, None) == 0
    assert L.boa_orthogonalize(None, P, 1, None) == EINVAL


def test_binding_refuses_host_tensors():
    with pytest.raises(ValueError, match="device"):
        boa.orthogonalize(torch.zeros(4, 5))
