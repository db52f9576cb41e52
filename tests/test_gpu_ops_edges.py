"""Query-tower operators on the GPU, at the edges of what a call may ask: single
gradients, probabilities next to 1, values next to the types' ends, many queries
of one point. Bounds add up what the formula's steps can do, as in
test_gpu_ops.py."""
import math

import pytest
import torch

import paper_2609_16175_amd as boa

from test_gpu_ops import BF16, EPS, F32, gen, sums, unit, xent_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("B,V,d", [(1, 500, 32), (20, 300, 112), (64, 900, 128), (90, 66_000, 16), (40, 700, 200)])
def test_softmax_xent_bias_gradient_alone(B, V, d, dt):
    # with few queries, or many points, one block has all of a point's queries
    h, pts, labels, bias = (t.cuda() for t in xent_case(B, V, d, dt, seed=B + V + d))
    whole = boa.softmax_xent_grad(h, pts, labels, bias, 4.0, bias_grad=True)
    r = boa.softmax_xent_grad(h, pts, labels, bias, 4.0, h_grad=False, rows_grad=False, bias_grad=True)
    assert r.dh is None and r.drows is None
    assert torch.equal(r.dbias, whole.dbias) and torch.equal(r.loss, whole.loss)
    r = boa.softmax_xent_grad(h, pts, labels, bias, 4.0, rows_grad=False, bias_grad=True)
    assert torch.equal(r.dbias, whole.dbias) and torch.equal(r.dh, whole.dh)
    bias.requires_grad_()
    boa.softmax_xent(h, pts, labels, bias, 4.0).backward()
    assert torch.equal(bias.grad, whole.dbias)
