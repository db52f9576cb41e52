"""Orthogonalised updates whose steps let singular values grow, on the GPU against
plain float64 computations, with the bounds of test_gpu_orth.py."""
import math

import pytest
import torch

import paper_2609_16175_amd as boa
import test_gpu_orth as updates
from test_gpu_orth import BF16, CO, F16, F32

pytestmark = pytest.mark.gpu


def one_direction(rows, cols, dt, value=0.3):
    """An update whose singular vectors are single coordinates: all of a singular value is in one value of X, X X^T, ..."""
    g = torch.zeros(rows, cols)
    g[rows // 2, cols // 3] = value
    return g.to(dt)


GROWING = [[(4.0, 0.0, 0.0), CO], [(7.9, 0.0, 0.0), CO], [(30.0, 0.0, 0.0), (1.5, -0.5, 0.0)], [(100.0, 0.0, 0.0), (0.25, 0.0, 0.125)],
           [(1.0, 40.0, 200.0), (1.0, 0.5, 0.0)], [(3.0, 0.0, 0.0)] * 9 + [(0.5, -0.25, 0.0)]]


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("co", GROWING)
@pytest.mark.parametrize("rows,cols", [(100, 120), (140, 129), (300, 70), (40, 1000), (20, 30)])
def test_singular_values_that_grow(rows, cols, co, dt):
    g = one_direction(rows, cols, dt)
    updates.check_all(g, boa.orthogonalize(g.cuda(), steps=len(co), coefficients=co), dt, co)
    g = updates.update(rows, cols, dt, rows + cols, 3).to(dt)
    updates.check_all(g, boa.orthogonalize(g.cuda(), steps=len(co), coefficients=co), dt, co)


@pytest.mark.parametrize("rows,cols", [(100, 120), (140, 129)])
def test_float16_up_to_its_range(rows, cols):
    g = one_direction(rows, cols, F16)
    co = [(4.0, 0.0, 0.0), CO]   # 1,789
    updates.check_all(g, boa.orthogonalize(g.cuda(), steps=2, coefficients=co), F16, co)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(100, 120), (140, 129)])
def test_singular_values_to_the_contract_s_end(rows, cols, dt):
    # 2^23, and a step that takes it back below 1
    co = [(2.0 ** 12, 0.0, 0.0), (2.0 ** 11, 0.0, 0.0), (2.0 ** -24, 0.0, 0.0), (1.5, -0.5, 0.0)]
    g = one_direction(rows, cols, dt)
    updates.check_all(g, boa.orthogonalize(g.cuda(), steps=4, coefficients=co), dt, co)
    co = co[:2] + [(0.0, 2.0 ** -50, 0.0), CO]
    updates.check_all(g, boa.orthogonalize(g.cuda(), steps=4, coefficients=co), dt, co)


def test_default_steps_keep_their_scales():
    # any number of the default steps: singular values stay below 1.21
    g = updates.update(130, 200, F32, 7)
    for steps in (6, 12, 32):
        got = boa.orthogonalize(g.cuda(), steps=steps)
        s = torch.linalg.svdvals(got.double().cpu())
        assert math.isfinite(float(s.max())) and 0.6 < float(s.min()) and float(s.max()) < 1.21
