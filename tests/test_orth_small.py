"""Which updates are orthogonalised in one block, in float32: those that take no
work memory (no GPU needed)."""
import pytest

from paper_2609_16175_amd import ops
from test_orth_refusals import _orth


@pytest.mark.parametrize("few,most", [(1, 2048), (16, 2048), (17, 1024), (32, 1024), (33, 672), (48, 672), (49, 480), (64, 480), (65, 0)])
def test_sizes_in_one_block(few, most):
    def takes(rows, cols):
        return ops._lib().boa_orthogonalize_workspace(ops.C.byref(_orth(rows=rows, cols=cols, update_stride=cols, update_batch=rows * cols)))

    for n in {max(few, most), most + 1 if most else few, 1 << 14}:
        for rows, cols in ((few, n), (n, few)):
            assert (takes(rows, cols) == 0) == (n <= most), (rows, cols)
