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


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("d", [64, 200])
@pytest.mark.parametrize("B", [20, 150])
def test_softmax_xent_probabilities_next_to_one(B, d, dt):
    # 1 - p of the label from above 1e-4 down to below 1e-9: gradients and losses keep the digits of 1 - p, whatever it is beside 1
    V = 400
    g = gen(B + d)
    pts = torch.randn(V, d, generator=g)
    pts = (pts / pts.norm(dim=1, keepdim=True)).to(dt)
    labels = torch.randperm(V, generator=g)[:B]
    h = (pts.float()[labels] * torch.linspace(14, 46, B)[:, None]).to(dt)
    bias = torch.zeros(V)
    H, C = h.double(), pts.double()
    l = H @ C.t()
    rows = torch.arange(B)
    own = l[rows, labels].clone()
    l[rows, labels] = -math.inf
    rest = torch.logsumexp(l, 1) - own                       # log of the others' sum over the label's
    lse = own + torch.log1p(torch.exp(rest))
    p = torch.exp(l - lse[:, None])                          # 0 at the label
    q = p.clone()
    q[rows, labels] = -torch.exp(rest + own - lse)           # p_label - 1
    left = -q[rows, labels]
    assert left.max() > 1e-4 and left.min() < 1e-9
    # relative error of an exponential: twice its logit's absolute one; then the sums', and rounding as an operand
    e_l = (sums(6 * d) + 8 * EPS) * (H.abs() @ C.abs().t()).amax(1, keepdim=True)
    e_p = 4 * e_l + sums(V) + 32 * EPS
    r = boa.softmax_xent_grad(h.cuda(), pts.cuda(), labels.cuda(), bias.cuda(), reduction="none", bias_grad=True)
    u = unit(dt)
    e_q = p * (e_p + u + sums(6 * V + 6 * B))
    e_q[rows, labels] = (left[:, None] * (e_p + sums(6 * V + 6 * B)))[:, 0]

    def near(got, want, bound):
        got = got.double().cpu()
        assert ((got - want).abs() <= 1.02 * bound).all(), float(((got - want).abs() / bound).max())

    loss = torch.log1p(torch.exp(rest))
    near(r.loss, loss, loss * (e_p[:, 0] + 8 * EPS))
    near(r.dh, q @ C, e_q @ C.abs() + u * (q @ C).abs())
    near(r.drows, q.t() @ H, e_q.t() @ H.abs() + u * (q.t() @ H).abs() + 1e-42)
    near(r.dbias, q.sum(0), (q.abs() * e_p).sum(0) + sums(B) * q.abs().sum(0) + 1e-42)
