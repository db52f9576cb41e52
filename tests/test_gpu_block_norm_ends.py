"""The norms around a residual block where values are not finite and where a
launch ends, on the GPU."""
import math

import pytest
import torch

import paper_2609_16175_amd as boa
from test_gpu_block_norm import BF16, F16, F32, call, case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("gate", [None, "features", "rows"])
@pytest.mark.parametrize("post,pre", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("d", [5, 96, 413, 1024, 4500, 9000])
def test_values_that_are_not_finite_without_dy(d, post, pre, gate, dt):
    # nothing comes back through the second norm: dx = scale dh whatever h is, and what f's rows give
    # is the same bits as with other values in the rows of x
    c = case(13, d, dt, dt, d, post=post, pre=pre, gate=gate) | {"dy": None}
    _, want = call(c)
    bad = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    bad["x"][2, d // 2], bad["x"][7, 0], bad["x"][9, d - 1] = math.inf, math.nan, -math.inf
    _, got = call(bad)
    for name, t in vars(want).items():
        assert t is None or torch.equal(getattr(got, name), t), name
    assert all(t is None or torch.isfinite(t).all() for t in vars(got).values())
    if pre:
        assert not got.dweight.any() and not got.dbias.any()
    # f's own row: its norm is not finite, but dx is; without that norm df neither asks what f is
    bad["f"][4, d // 3] = math.nan
    bad["f"][6, 1] = math.inf
    _, got = call(bad)
    assert torch.equal(got.dx, want.dx)
    rows = lambda t: (~torch.isfinite(t)).any(1).cpu().nonzero().flatten().tolist()  # noqa: E731
    if post:
        assert rows(got.df) == [4, 6]
    else:
        assert torch.equal(got.df, want.df)
    if gate == "rows":
        assert rows(got.dgate) == [4, 6]
    elif gate == "features":
        # a norm spreads them over its row
        spoilt = (~torch.isfinite(got.dgate)).cpu().nonzero().flatten().tolist()
        assert spoilt == (list(range(d)) if post else sorted({d // 3, 1}))


@pytest.mark.parametrize("d", [4104, 8192])
def test_more_rows_than_a_launch_with_512_threads_a_row_takes(d):
    # a block of 512 threads a row: 2^22 rows a launch; only the residual sum, of x with itself
    rows = (1 << 23) + 5 if d == 4104 else (1 << 22) + 5
    x = torch.empty(rows, d, device="cuda", dtype=BF16)
    x.view(torch.int16).fill_(0x3F80)   # ones
    at = sorted({0, (1 << 22) - 1, 1 << 22, (1 << 22) + 4, rows - 1})
    g = torch.Generator().manual_seed(1)
    some = torch.randn(len(at), d, generator=g).bfloat16()
    x[at] = some.cuda()
    h, y, stats = boa.block_norm_forward(x, x, pre=False, scale=0.5)
    assert y is None
    assert torch.equal(h[at].cpu(), (some.float() * 1.5).bfloat16())
    for lo in range(0, rows, 1 << 20):   # every other row was written, too
        assert int((h[lo:lo + (1 << 20), ::512] == 1.5).sum(1).eq(h[:1, ::512].numel()).sum()) >= min(rows - lo, 1 << 20) - len(at)
