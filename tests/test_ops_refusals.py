"""Query-tower operators: arguments the C interface refuses, with its codes and
messages, before any device work (no GPU needed), and the binding's checks."""
import ctypes as C

import pytest
import torch

import paper_2609_16175_amd as boa
from paper_2609_16175_amd import ops

EINVAL, EUNSUPPORTED = -1, -4
P = 4096   # stands for a device pointer: refused calls never read it


def _err():
    return boa.lib().boa_last_error().decode()


def _norm(**over):
    a = dict(x=P, rows=4, d=16, stride=16, dtype=0, w=P, b=P, pd=0, eps=1e-5, y=P, mean=P, rstd=P)
    a.update(over)
    return ops._lib().boa_layer_norm(a["x"], a["rows"], a["d"], a["stride"], a["dtype"], a["w"], a["b"], a["pd"], a["eps"],
                                     a["y"], a["mean"], a["rstd"], None)


@pytest.mark.parametrize("over,needle", [
    (dict(dtype=7), "dtype"), (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"), (dict(d=0), "d out of range"),
    (dict(d=(1 << 20) + 1), "d out of range"), (dict(stride=15), "stride"), (dict(x=None), "NULL"), (dict(y=None), "NULL"),
    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(pd=1), "parameters"),
])
def test_layer_norm_refuses(over, needle):
    assert _norm(**over) == EINVAL and needle in _err()


def test_layer_norm_of_nothing_is_fine():
    assert _norm(rows=0, x=None, y=None) == 0


def _norm_back(**over):
    a = dict(dy=P, dys=16, x=P, xs=16, rows=4, d=16, dtype=0, w=P, pd=0, mean=P, rstd=P, dx=P, dw=P, db=P, ws=P, n=1 << 20)
    a.update(over)
    return ops._lib().boa_layer_norm_backward(*a.values(), None)


@pytest.mark.parametrize("over,needle", [
    (dict(dy=None), "NULL"), (dict(mean=None), "NULL"), (dict(dys=3), "stride"), (dict(ws=None), "workspace"),
    (dict(n=8), "workspace"), (dict(ws=P + 4), "workspace"), (dict(dtype=3), "dtype"), (dict(xs=1), "stride"),
])
def test_layer_norm_backward_refuses(over, needle):
    assert _norm_back(**over) == EINVAL and needle in _err()


def _xent(grad=False, ws=P, n=1 << 40, **over):
    a = ops.Xent(dtype=0, d=32, B=4, V=100, h=P, h_stride=32, points=P, points_stride=32, labels=P, bias=None, scale=1.0,
                 reduction=2, loss=P)
    for k, v in over.items():
        setattr(a, k, v)
    L = ops._lib()
    return (L.boa_softmax_xent_grad if grad else L.boa_softmax_xent)(C.byref(a), ws, n, None)


@pytest.mark.parametrize("over,code,needle", [
    (dict(dtype=2), EUNSUPPORTED, "float16"), (dict(dtype=9), EINVAL, "dtype"), (dict(d=0), EINVAL, "d out of range"),
    (dict(d=4097), EINVAL, "d out of range"), (dict(B=-1), EINVAL, "B out of range"), (dict(V=0), EINVAL, "V out of range"),
    (dict(V=1 << 31), EINVAL, "V out of range"), (dict(h_stride=31), EINVAL, "stride"),
    (dict(points_stride=31), EINVAL, "stride"), (dict(reduction=3), EINVAL, "reduction"),
    (dict(scale=float("inf")), EINVAL, "scale"), (dict(h=None), EINVAL, "NULL"), (dict(points=None), EINVAL, "NULL"),
    (dict(labels=None), EINVAL, "NULL"), (dict(loss=None), EINVAL, "loss"), (dict(ws=None), EINVAL, "workspace"),
    (dict(ws=P + 8), EINVAL, "workspace"), (dict(n=16), EINVAL, "workspace"),
    (dict(grad=True, dbias=P), EINVAL, "bias"), (dict(grad=True, n=64), EINVAL, "workspace"),
])
def test_softmax_xent_refuses(over, code, needle):
    assert _xent(**over) == code and needle in _err()


def test_softmax_xent_refuses_more_queries_than_its_launches_take():
    assert _xent(B=(1 << 21) + 1) == EINVAL and "B out of range" in _err()
    assert _xent(B=1 << 21, n=16) == EINVAL and "workspace" in _err()


def test_xent_null_struct():
    assert ops._lib().boa_softmax_xent(None, P, 1 << 30, None) == EINVAL
    assert ops._lib().boa_softmax_xent_workspace(None, 1) == EINVAL


def test_xent_workspace_grows_with_what_is_asked():
    a = ops.Xent(dtype=1, d=128, B=512, V=1_000_000, h=P, h_stride=128, points=P, points_stride=128, labels=P, scale=1.0,
                 reduction=2, loss=P)
    L = ops._lib()
    loss = L.boa_softmax_xent_workspace(C.byref(a), 0)
    a.dh = P
    one = L.boa_softmax_xent_workspace(C.byref(a), 1)
    a.dpoints = P
    two = L.boa_softmax_xent_workspace(C.byref(a), 1)
    assert 0 < loss < one < two
    # far below the logits' 2 GB
    assert two < 512 * 1_000_000 * 4 // 2


def _matvec(**over):
    a = dict(x=P, M=2, xs=64, dtype=1, codes=P, rows=10, K=64, cs=32, s=P, o=P, ss=2, sd=1, group=32, y=P, ys=10)
    a.update(over)
    return ops._lib().boa_matvec_fourbit(*a.values(), None)


@pytest.mark.parametrize("over,needle", [
    (dict(dtype=5), "dtype"), (dict(sd=5), "dtype"), (dict(M=-1), "M out of range"), (dict(M=65536), "M out of range"),
    (dict(rows=-1), "rows"), (dict(K=0), "K out of range"), (dict(K=(1 << 20) + 1), "K out of range"), (dict(group=0), "group"),
    (dict(cs=31), "codes"), (dict(ss=1), "scales"), (dict(xs=63), "stride"), (dict(ys=9), "stride"), (dict(x=None), "NULL"),
    (dict(codes=None), "NULL"), (dict(s=None), "NULL"), (dict(y=None), "NULL"),
])
def test_matvec_refuses(over, needle):
    assert _matvec(**over) == EINVAL and needle in _err()


def test_matvec_of_nothing_is_fine():
    assert _matvec(M=0, x=None, y=None) == 0 and _matvec(rows=0, codes=None) == 0


def test_binding_refuses_host_tensors():
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError, match="device"):
        boa.layer_norm_forward(x)
    with pytest.raises(ValueError, match="device"):
        boa.softmax_xent(x, x, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="device"):
        boa.matvec_4bit(x, torch.zeros(3, 4, dtype=torch.uint8), torch.ones(3, 1))


def test_unknown_attribute():
    with pytest.raises(AttributeError):
        boa.no_such_operator


@pytest.mark.parametrize("grad", [0, 1])
@pytest.mark.parametrize("dtype,B,V,d", [(1, 1, 4_000_000, 1001), (0, 40, 500_000, 4096), (0, 33, 3_000_000, 768),
                                         (1, 20, 3_000_000, 2000)])
def test_xent_workspace_copies_two_gigabytes_of_points_at_most(dtype, B, V, d, grad):
    # points that are not read in place are copied in pieces; these are of odd widths or alignment, or float32
    a = ops.Xent(dtype=dtype, d=d, B=B, V=V, h=P, h_stride=d, points=P + 8, points_stride=d, labels=P, bias=P, scale=1.0,
                 reduction=2, loss=P)
    if grad:
        a.dh = a.dpoints = a.dbias = P
    L = ops._lib()
    # beside the copy: up to 256 MB of probabilities, shares of the queries' gradient, biases and first queries of the points
    beside = (1 << 28) + 512 * 128 * (d + 16) * 4 + 8 * V if grad else 1 << 26
    assert 0 < L.boa_softmax_xent_workspace(C.byref(a), grad) <= (1 << 31) + beside


def test_error_buffer_is_written_in_one_place():
    # the thread's buffer and its size belong to one source; the operators hand their messages over
    import glob
    import os
    from paper_2609_16175_amd import build
    sources = {os.path.basename(f): open(f).read() for f in glob.glob(os.path.join(build.PKG, "csrc", "*"))}
    assert [f for f, s in sources.items() if "g_err" in s] == ["boa_api.hip"]
    assert not [f for f, s in sources.items() if "boa_last_error()" in s.replace("for boa_last_error()", "")]
    # a message longer than most arrives whole
    assert _xent(dtype=2) == EUNSUPPORTED and _err().endswith("use bfloat16 or float32")


def test_layer_norm_backward_workspace_is_bounded():
    ws = ops._lib().boa_layer_norm_backward_workspace
    assert ws(8, 768) == 2 * 768 * 4 and ws(1 << 20, 8192) == 1024 * 2 * 8192 * 4
    for d in (1, 4096, 16_384, 16_385, 100_000, 1 << 20):
        for rows in (0, 1, 9, 1 << 13, (1 << 31) - 1):
            assert 0 < ws(rows, d) <= max(2 * d * 4, 1 << 27)
