"""Linear layers at the ends of their ranges, on the GPU against plain float64
computations: pre-activations next to 0, gelu far below 0.

`unit`, `tiny`, `within` and the bound of a product's sums are those of
test_gpu_linear.py.
"""
import math

import pytest
import torch

import paper_2609_16175_amd as boa
import test_gpu_linear as linears
from test_gpu_linear import BF16, EPS, F16, F32, product_error, sums, tiny, unit, within

pytestmark = pytest.mark.gpu


def check_relu(x, w, b, dt, y, dy, grads):
    """A slope is 0 or 1 by the sign of the float32 z: free only where z is
    within its own sum's error of 0, whatever z is kept in. dz is dy or 0 then,
    which no type rounds."""
    X, W, D = x.double(), w.double(), dy.double()
    z = X @ W.T + (0 if b is None else b.double())
    e_z = product_error(X, W, dt) + 2 * EPS * (z.abs() + (0 if b is None else b.double().abs()))
    within(y, z.clamp(min=0), 1.01 * (unit(dt) * z.clamp(min=0) + e_z) + tiny(dt), "y")
    dz = D * (z > 0)
    e_d = D.abs() * (z.abs() <= e_z)
    Z = dz.abs() + e_d
    dx, dw, db = grads
    want, e = dz @ W, e_d @ W.abs() + product_error(Z, W.abs().T.contiguous(), dt)
    within(dx, want, 1.01 * (unit(dt) * (want.abs() + e) + e) + tiny(dt), "dx")
    want, e = dz.T @ X, e_d.T @ X.abs() + product_error(Z.T.contiguous(), X.abs().T.contiguous(), dt)
    within(dw, want, 1.01 * (unit(dt) * (want.abs() + e) + e) + tiny(dt), "dw")
    want = dz.sum(0)
    within(db, want, 1.01 * (unit(dt) * want.abs() + e_d.sum(0) + sums(len(x)) * dz.abs().sum(0)) + tiny(dt), "db")


# x and w scaled so that z lies far below float16's smallest value, or (float16) around it
SMALL = [(BF16, 1e-6, 1e-6), (BF16, 1e-18, 1e-12), (F16, 2.0 ** -10, 2.0 ** -17), (F32, 1e-6, 1e-6), (F32, 1e-12, 1e-18)]


@pytest.mark.parametrize("dt,by_x,by_w", SMALL)
@pytest.mark.parametrize("M,N,K", [(1, 24, 40), (5, 33, 64), (40, 130, 72), (200, 96, 100), (300, 77, 2100)])
def test_relu_of_small_values(M, N, K, dt, by_x, by_w):
    x, w, _, _, dy = linears.case(M, N, K, dt, M + K)
    x, w = (x.double() * by_x).to(dt), (w.double() * by_w).to(dt)
    y, pre = boa.linear_forward(x.cuda(), w.cuda(), activation="relu", keep=True)
    grads = boa.linear_backward(dy.cuda(), x.cuda(), w.cuda(), pre, activation="relu")
    check_relu(x, w, None, dt, y, dy, grads)
    assert grads[2].abs().max() > 0


def test_relu_of_one_small_value():
    for dt in (BF16, F16, F32):
        for M in (1, 70):
            for value in (6e-8, 2.0 ** -25, 2.0 ** -26, 1e-9, 1e-30):
                if dt == F16 and value < 2.0 ** -14:   # of two factors that float16 has
                    x, w = torch.full((M, 1), 2.0 ** -12, dtype=dt), torch.full((1, 1), value * 2.0 ** 12).to(dt)
                else:
                    x, w = torch.full((M, 1), value, dtype=dt), torch.ones(1, 1, dtype=dt)
                up = float(x[0, 0]) * float(w[0, 0]) > 0
                y, pre = boa.linear_forward(x.cuda(), w.cuda(), activation="relu", keep=True)
                dx, dw, db = boa.linear_backward(torch.ones_like(y), x.cuda(), w.cuda(), pre, activation="relu")
                assert torch.equal(dx.cpu(), w[0, 0].expand(M, 1) if up else torch.zeros(M, 1, dtype=dt)), (dt, M, value)
                assert float(db) == (M if up else 0)
                _, pre = boa.linear_forward(-x.cuda(), w.cuda(), activation="relu", keep=True)
                assert not boa.linear_backward(torch.ones_like(y), x.cuda(), w.cuda(), pre, activation="relu")[0].any()


@pytest.mark.parametrize("dt,by_x,by_w", SMALL)
@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
def test_activations_of_small_values(kind, dt, by_x, by_w):
    # y is z / 2 to z's own relative size: the share of z^2 is below 2^-20
    for M in (5, 200):
        x, w, _, _, dy = linears.case(M, 96, 100, dt, M)
        x, w = (x.double() * by_x).to(dt), (w.double() * by_w).to(dt)
        y, pre = boa.linear_forward(x.cuda(), w.cuda(), activation=kind, keep=True)
        X, W = x.double(), w.double()
        z = X @ W.T
        e = product_error(X, W, dt) + 2.0 ** -18 * z.abs()
        within(y, z / 2, 1.01 * (unit(dt) * z.abs() / 2 + e) + tiny(dt), kind)
        grads = boa.linear_backward(dy.cuda(), x.cuda(), w.cuda(), pre, activation=kind)
        linears.check(x, w, None, None, kind, dt, None, dy, grads, dt)


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("M", [16, 640])
def test_gelu_far_below_zero(M, dt):
    """Held relative to the values. z is exact: one product, with 1. The
    distribution and its density are good to 2^-21 and some roundings of
    themselves, 2^-20 in all; in 16 bits to 2^-14, z^2 2^-22 for the roundings of
    the density's exponent, and 2^-18 for the rest. The slope is rounded to the
    layer's type as dz, and dx, its product with 1, is the same value."""
    values = (-torch.arange(2 * 64, 12 * 64, dtype=torch.float64) / 64).to(dt)
    w = torch.ones(1, 1, dtype=dt)
    for x in values[:, None].split(M):
        z = x.double()
        y, pre = boa.linear_forward(x.cuda(), w.cuda(), activation="gelu", keep=True)
        off = 2.0 ** -20 if dt == F32 else z * z * 2.0 ** -22 + 2.0 ** -14 + 2.0 ** -18
        below = 0.5 * torch.special.erfc(-z / math.sqrt(2))   # torch's ndtr is 1 + erf, which cancels
        want = z * below
        within(y, want, 1.01 * (unit(dt) + off) * want.abs() + tiny(dt), "y")
        dx, _, _ = boa.linear_backward(torch.ones_like(y), x.cuda(), w.cuda(), pre, activation="gelu", need=(True, False, False))
        other = z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        want = below + other
        within(dx, want, 1.01 * (unit(dt) * want.abs() + off * (below + other.abs())) + tiny(dt), "dx")
