"""4-bit rows: codes, scales and offsets against their definition (CPU)."""
import pytest
import torch

from workloads import rows4


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,K,group", [(1, 32, 32), (5, 64, 32), (7, 96, 16), (3, 8, 2)])
def test_quantize(N, K, group, dtype):
    w = torch.randn(N, K, generator=torch.Generator().manual_seed(N * K))
    codes, s, o = rows4.quantize(w, group, dtype)
    assert codes.shape == (N, K // 2) and codes.dtype == torch.uint8 and s.shape == o.shape == (N, K // group)
    back = rows4.dequantize(codes, s, o)
    # half a step, and where scale and offset are rounded to bfloat16, what that moves the end of the range
    step = s.float().repeat_interleave(group, 1)
    slack = 0 if dtype == torch.float32 else 2.0 ** -7 * (w.abs().max() + 15 * step)
    assert ((back - w).abs() <= 0.5 * step * 1.001 + 1e-6 + slack).all()
    # nibble order
    q = torch.stack((codes & 15, codes >> 4), 2).reshape(N, K)
    assert torch.equal(rows4.dequantize(codes, torch.ones_like(s), torch.zeros_like(o)), q.float())


def test_quantize_constant_rows_and_refusals():
    codes, s, o = rows4.quantize(torch.full((2, 32), 1.5), 32)
    assert not codes.any() and torch.equal(rows4.dequantize(codes, s, o), torch.full((2, 32), 1.5))
    with pytest.raises(ValueError):
        rows4.quantize(torch.zeros(2, 33), 32)
