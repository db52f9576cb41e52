"""Linear layers with their epilogue on the GPU against plain float64 computations.

Tolerances are bounds, not fits: `unit(type)` is the largest relative error of
one rounding to a type; a float32 sum of n terms held in lanes or matrix
instructions is off by at most (n / 16 + 32) roundings of its terms'
magnitudes; each check adds up what the formula's steps can do.
"""
import math

import pytest
import torch

import paper_2609_16175_amd as boa

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = 2.0 ** -24
ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")


def unit(dt):
    return {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}[dt]


def tiny(dt):   # half the smallest denormal's spacing
    return {F32: 0.0, BF16: 0.0, F16: 2.0 ** -25}[dt]


def sums(n):
    return (n / 16 + 32) * EPS


def within(got, want, bound, what=""):
    got = got.detach().double().cpu()
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), what
    over = (got - want).abs() - bound
    assert (over <= 0).all(), f"{what}: off by {float((got - want).abs().max()):.3g}, {float(over.max()):.3g} over the bound"


def gen(seed):
    return torch.Generator().manual_seed(seed)


def act(z, kind):
    if kind == "relu":
        return z.clamp(min=0)
    if kind == "silu":
        return z * torch.sigmoid(z)
    if kind == "gelu":
        return z * torch.special.ndtr(z)
    if kind == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def slope(z, kind):
    if kind == "relu":
        return (z > 0).double()
    if kind == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    if kind == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def product_error(a, b, dt):
    """Of a @ b.T, a and b as the product has them: the sums, and in float32 the
    operands' parts: 2^-22 of each value, or 2^-40 of its row's largest (a
    product of the two roundings, and the parts' product left out, below that)."""
    n = a.shape[1]
    A, B = a.abs(), b.abs()
    e = sums(n * (3 if dt == F32 else 1)) * (A @ B.T)
    if dt == F32:
        top_a, top_b = A.amax(1, keepdim=True), B.amax(1, keepdim=True)
        e = e + 2.0 ** -20.9 * (A @ B.T) + 2.0 ** -39 * (top_a * B.sum(1)[None] + A.sum(1, keepdim=True) * top_b.T)
    return e


def check(x, w, b, r, kind, dt, y=None, dy=None, grads=None, db_dt=None):
    X, W = x.double(), w.double()
    bias = 0 if b is None else b.double()
    z = X @ W.T + bias
    e_z = product_error(X, W, dt) + 2 * EPS * (z.abs() + (0 if b is None else b.double().abs()))
    # the activations: slopes of at most 1.13, a few roundings, and in 16 bits exponentials good to 2^-20
    fine = 16 * EPS if dt == F32 else 2.0 ** -19
    if y is not None:
        want = act(z, kind)
        e_y = 1.13 * e_z + (0 if kind in ("none", "relu") else fine * z.abs() + fine * 1e-3)
        if r is not None:
            want = want + r.double()
            e_y = e_y + EPS * want.abs()
        within(y, want, 1.01 * (unit(dt) * want.abs() + e_y) + tiny(dt), "y")
    if grads is None:
        return
    dx, dw, db = grads
    D = dy.double()
    dz = D * slope(z, kind)
    kept = e_z if dt == F32 else e_z + 2.0 ** -11 * z.abs() + 2.0 ** -25
    if kind == "none":
        e_s = torch.zeros_like(z)
    elif kind == "relu":
        e_s = (z.abs() <= kept).double()
    else:   # |second derivatives| are below 1.1; the slope's own evaluation
        e_s = 1.1 * kept + 4 * fine * (1 + z.abs())
    e_f = D.abs() * e_s + 2 * EPS * dz.abs()
    if db is not None:
        within(db, dz.sum(0), 1.01 * (unit(db_dt) * dz.sum(0).abs() + e_f.sum(0) + sums(len(x)) * dz.abs().sum(0)) + tiny(db_dt), "db")
    e_d = e_f if dt == F32 or kind == "none" else e_f + 1.01 * unit(dt) * (dz.abs() + e_f) + tiny(dt)
    Z = dz.abs() + e_d
    if dx is not None:
        want = dz @ W
        e = e_d @ W.abs() + product_error(Z, W.abs().T.contiguous(), dt)
        within(dx, want, 1.01 * (unit(dt) * (want.abs() + e) + e) + tiny(dt), "dx")
    if dw is not None:
        want = dz.T @ X
        e = e_d.T @ X.abs() + product_error(Z.T.contiguous(), X.abs().T.contiguous(), dt)
        within(dw, want, 1.01 * (unit(dt) * (want.abs() + e) + e) + tiny(dt), "dw")


def case(M, N, K, dt, seed, bias=None, residual=False, gap=0):
    g = gen(seed)
    x = torch.randn(M, K + gap, generator=g).to(dt)[:, :K]
    w = (torch.randn(N, K + gap, generator=g) / math.sqrt(K)).to(dt)[:, :K]
    b = None if bias is None else (0.3 * torch.randn(N, generator=g)).to(bias)
    r = torch.randn(M, N + gap, generator=g).to(dt)[:, :N] if residual else None
    dy = torch.randn(M, N + gap, generator=g).to(dt)[:, :N]
    return x, w, b, r, dy


def cu(t):   # with its strides
    if t is None:
        return None
    wide = torch.zeros(t.shape[0], t.stride(0), dtype=t.dtype) if t.dim() == 2 and t.shape[0] > 1 else None
    if wide is None or t.stride(0) == t.shape[1]:
        return t.cuda()
    wide = torch.full((t.shape[0], t.stride(0)), 7.0, dtype=t.dtype, device="cuda")
    wide[:, :t.shape[1]] = t.cuda()
    return wide[:, :t.shape[1]]


def both(M, N, K, dt, seed, kind, bias=None, residual=False, gap=0):
    x, w, b, r, dy = case(M, N, K, dt, seed, bias, residual, gap)
    xc, wc, bc, rc, dyc = (cu(t) for t in (x, w, b, r, dy))
    y, pre = boa.linear_forward(xc, wc, bc, residual=rc, activation=kind, keep=True)
    assert y.dtype == dt and (pre is None) == (kind == "none")
    db_dt = dt if bias is None else bias
    grads = boa.linear_backward(dyc, xc, wc, pre, activation=kind, bias_dtype=db_dt)
    assert grads[0].dtype == grads[1].dtype == dt and grads[2].dtype == db_dt
    check(x, w, b, r, kind, dt, y, dy, grads, db_dt)
    return (xc, wc, bc, rc, dyc), (y, pre, grads)


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 768, 768), (2, 5, 3), (3, 17, 31), (5, 16, 33), (13, 100, 64), (16, 24, 40),
                                   (17, 9, 1000), (33, 130, 72), (63, 64, 65), (64, 40, 129), (65, 33, 8), (128, 256, 128),
                                   (129, 257, 136), (200, 264, 1000), (257, 129, 413), (300, 77, 63), (1000, 96, 264), (2051, 40, 24)])
def test_linear(M, N, K, dt):
    both(M, N, K, dt, M * 7 + N * 3 + K, ACTS[(M + N) % 5], bias=(None, dt, F32)[K % 3], residual=M % 2 == 1)


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("M,N,K", [(1, 33, 4100), (16, 48, 4100), (17, 48, 4100), (33, 40, 1500), (48, 4100, 64), (64, 17, 777), (64, 24, 3),
                                   (65, 33, 1024), (100, 40, 515), (128, 24, 520), (129, 24, 520), (2048, 64, 40), (2049, 64, 40),
                                   (1024, 100, 72), (1025, 100, 72)])
def test_where_the_kernels_change(M, N, K, dt):
    # few rows and many (by rows, k and type), both gradients in one launch and in two
    both(M, N, K, dt, M + N + K, "gelu_tanh", bias=dt, residual=True)


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("M", [4, 70, 300])
def test_activations(M, kind, dt):
    both(M, 120, 88, dt, M, kind, bias=F32, residual=True)


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("M,N,K,gap", [(3, 40, 48, 8), (90, 64, 56, 8), (90, 64, 56, 3), (513, 65, 71, 1), (40, 33, 47, 5)])
def test_strided_rows(M, N, K, gap, dt):
    both(M, N, K, dt, M + gap, "gelu", bias=dt, residual=True, gap=gap)
    both(M, N, K, dt, M + gap, "none", bias=None, residual=False, gap=gap)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("M,N,K", [(700, 520, 776), (3000, 264, 520), (520, 1100, 2100), (9000, 72, 40)])
def test_many_tiles_and_splits(M, N, K, dt):
    both(M, N, K, dt, K, "silu", bias=dt)


def test_tile_shapes_each():
    # 256, 128 and 64 rows a tile: the sizes at which the cut changes, by blocks and by length of the sum
    both(4096, 2048, 64, BF16, 1, "none")
    both(2048, 1024, 136, BF16, 2, "relu", bias=BF16)


@pytest.mark.parametrize("dt", [F32, BF16, F16])
def test_same_bits_again(dt):
    t, (y, pre, grads) = both(700, 136, 1000, dt, 5, "gelu", bias=dt, residual=True)
    xc, wc, bc, rc, dyc = t
    for _ in range(2):
        y2, pre2 = boa.linear_forward(xc, wc, bc, residual=rc, activation="gelu", keep=True)
        g2 = boa.linear_backward(dyc, xc, wc, pre2, activation="gelu")
        assert torch.equal(y, y2) and torch.equal(pre, pre2) and all(torch.equal(a, b) for a, b in zip(grads, g2))


@pytest.mark.parametrize("dt", [F32, BF16, F16])
def test_no_rows(dt):
    x, w = torch.empty(0, 24, device="cuda", dtype=dt), torch.ones(10, 24, device="cuda", dtype=dt)
    y, pre = boa.linear_forward(x, w, activation="silu", keep=True)
    assert y.shape == pre.shape == (0, 10)
    dx, dw, db = boa.linear_backward(y, x, w, pre, activation="silu")
    assert dx.shape == (0, 24) and torch.equal(dw, torch.zeros_like(w)) and torch.equal(db, torch.zeros_like(db))


def test_needed_gradients_only():
    x, w, b, r, dy = case(100, 48, 40, BF16, 3, BF16)
    xc, wc, dyc = x.cuda(), w.cuda(), dy.cuda()
    whole = boa.linear_backward(dyc, xc, wc)
    for need in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 0, 0)):
        got = boa.linear_backward(dyc, xc, wc, need=need)
        assert all((a is None) == (not n) and (a is None or torch.equal(a, b)) for a, b, n in zip(got, whole, need))


@pytest.mark.parametrize("M", [5, 100])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_nan_stays_in_its_row(M, dt):
    x, w, b, _, dy = case(M, 72, 80, dt, 9, dt)
    x[2, 5] = math.nan
    x[4, 7] = math.inf
    y, pre = boa.linear_forward(x.cuda(), w.cuda(), b.cuda(), activation="relu" if M > 50 else "none", keep=True)
    bad = (~torch.isfinite(y)).any(1).cpu()
    assert bad[2] and bad[4] and bad.sum() == 2
    dy[3, 6] = math.nan
    dx, dw, db = boa.linear_backward(dy.cuda(), torch.zeros(M, 80, dtype=dt, device="cuda"), w.cuda())
    assert (~torch.isfinite(dx)).any(1).cpu().nonzero().flatten().tolist() == [3]
    assert (~torch.isfinite(dw)).any(1).cpu().nonzero().flatten().tolist() == [6]
    assert torch.isnan(db).cpu().nonzero().flatten().tolist() == [6]


def test_float32_keeps_rows_of_every_size():
    # each row and column has a scale of its own
    x, w, _, _, dy = case(100, 64, 96, F32, 4)
    x *= torch.logspace(-30, 30, 100)[:, None]
    w *= torch.logspace(-4, 4, 64)[:, None]
    y, _ = boa.linear_forward(x.cuda(), w.cuda())
    check(x, w, None, None, "none", F32, y)
    x, w, _, _, dy = case(100, 64, 96, F32, 4)
    x *= torch.logspace(-15, 15, 96)
    dy *= torch.logspace(-15, 15, 64)
    dx, dw, db = boa.linear_backward(dy.cuda(), x.cuda(), w.cuda())
    check(x, w, None, None, "none", F32, None, dy, (None, dw, db), F32)


def test_saturated_activations():
    # far from zero, where float16 ends too
    for kind in ACTS[1:]:
        z = torch.tensor([-3e38, -1e5, -65504.0, -200.0, -30.0, 0.0, 30.0, 200.0, 65504.0, 1e5, 3e38])
        for dt in (F32, BF16):
            x = z.to(dt)[:, None].repeat(8, 1).contiguous()
            w = torch.ones(3, 1, dtype=dt)
            y, pre = boa.linear_forward(x.cuda(), w.cuda(), activation=kind, keep=True)
            want = torch.where(x > 0, x, torch.zeros_like(x)).double().expand(-1, 3)
            within(y, want, 1e-9 + 2.0 ** -20 * want, kind)
            dx, _, _ = boa.linear_backward(torch.ones_like(y), x.cuda(), w.cuda(), pre, activation=kind)
            want = 3 * slope(z.to(dt).double().clamp(-40, 40), kind)[:, None].repeat(8, 1)
            within(dx, want, 1e-9 + 2.0 ** -7 * want.abs(), kind)


@pytest.mark.parametrize("kind", ["gelu", "none"])
def test_autograd(kind):
    x, w, b, r, dy = case(90, 40, 56, F32, 11, F32, True)
    leaves = [t.cuda().requires_grad_() for t in (x.reshape(9, 10, 56), w, b, r.reshape(9, 10, 40))]
    y = boa.linear(*leaves, activation=kind)
    assert y.shape == (9, 10, 40)
    y.backward(dy.cuda().reshape(9, 10, 40))
    check(x, w, b, r, kind, F32, y.reshape(90, 40), dy, (leaves[0].grad.reshape(90, 56), leaves[1].grad, leaves[2].grad), F32)
    assert torch.equal(leaves[3].grad.cpu().reshape(90, 40), dy)
    with torch.no_grad():
        assert torch.equal(boa.linear(*leaves, activation=kind), y)
    # the same tensor as input and residual: both gradients arrive
    x2 = torch.randn(70, 48, device="cuda", requires_grad=True)
    w2 = torch.randn(48, 48, device="cuda")
    boa.linear(x2, w2, residual=x2).sum().backward()
    want = (1 + w2.double().sum(0)).cpu().expand(70, 48)
    within(x2.grad, want, 1e-3 * torch.ones_like(want), "shared input")


@pytest.mark.parametrize("kind", ACTS[2:])
def test_gradient_against_differences(kind):
    x, w, b, _, dy = case(80, 24, 40, F32, 21, F32)
    y, pre = boa.linear_forward(x.cuda(), w.cuda(), b.cuda(), activation=kind, keep=True)
    dx, dw, db = boa.linear_backward(dy.cuda(), x.cuda(), w.cuda(), pre, activation=kind)
    f = lambda x_, w_, b_: float((act(x_ @ w_.T + b_, kind) * dy.double()).sum())  # noqa: E731
    X, W, Bs = x.double(), w.double(), b.double()
    g = gen(2)
    h = 1e-4   # central differences: the third derivative's share is h^2 of the value, float64's 1e-12 / h
    for grad, at in ((dx, 0), (dw, 1), (db, 2)):
        d = torch.randn(grad.shape, generator=g, dtype=torch.float64)
        args = [X, W, Bs]
        up, down = list(args), list(args)
        up[at], down[at] = args[at] + h * d, args[at] - h * d
        want = (f(*up) - f(*down)) / (2 * h)
        got = float((grad.double().cpu() * d).sum())
        scale = float((grad.double().cpu() * d).abs().sum())
        assert abs(got - want) <= 1e-5 * scale


def test_another_stream():
    x, w, b, r, dy = case(150, 72, 80, BF16, 6, BF16, True)
    xc, wc, bc, rc, dyc = (t.cuda() for t in (x, w, b, r, dy))
    want = boa.linear_forward(xc, wc, bc, rc, "silu", keep=True)
    wg = boa.linear_backward(dyc, xc, wc, want[1], "silu")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = boa.linear_forward(xc, wc, bc, rc, "silu", keep=True, stream=s)
    gg = boa.linear_backward(dyc, xc, wc, got[1], "silu", stream=s)
    s.synchronize()
    assert all(torch.equal(a, c) for a, c in zip((*want, *wg), (*got, *gg)))


@pytest.mark.parametrize("dt", [F32, BF16])
def test_captured(dt):
    x, w, b, r, dy = case(600, 136, 100, dt, 8, dt, True)
    xc, wc, bc, rc, dyc = (t.cuda() for t in (x, w, b, r, dy))

    def step():
        y, pre = boa.linear_forward(xc, wc, bc, rc, "gelu", keep=True)
        return (y, *boa.linear_backward(dyc, xc, wc, pre, "gelu"))

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for k in range(3):
        xc.copy_(torch.randn(x.shape, generator=gen(k)).to(dt))
        g.replay()
        got = [t.clone() for t in out]
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, step()))


def test_offsets_pass_32_bits():
    # outputs of 2^31 values and more: the last rows, checked on their own
    M, N, K = 1_060_000, 2048, 64
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.randn(M, K, device="cuda", generator=g).bfloat16()
    w = (torch.randn(N, K, device="cuda", generator=g) / 8).bfloat16()
    y, pre = boa.linear_forward(x, w, activation="relu", keep=True)
    for at in (slice(0, 100), slice(M // 2, M // 2 + 100), slice(M - 100, M)):
        check(x[at].cpu(), w.cpu(), None, None, "relu", BF16, y[at])
    dx, dw, db = boa.linear_backward(y, x, w, pre, activation="relu", need=(True, False, False))
    at = slice(M - 100, M)
    check(x[at].cpu(), w.cpu(), None, None, "relu", BF16, None, y[at].cpu(), (dx[at], None, None), BF16)


def test_more_tiles_than_a_launch_takes():
    # 2^24 tiles of 64 rows and more, 2^23 a launch
    M, N, K = (1 << 30) + 100, 1, 8
    g = torch.Generator("cuda").manual_seed(2)
    x = torch.empty(M, K, device="cuda", dtype=BF16).normal_(generator=g)
    w = torch.randn(N, K, device="cuda", generator=g).bfloat16()
    y, _ = boa.linear_forward(x, w)
    dx, _, _ = boa.linear_backward(y, x, w, need=(True, False, False))
    for at in (slice(0, 100), slice((1 << 29) - 50, (1 << 29) + 50), slice(M - 200, M)):
        check(x[at].cpu(), w.cpu(), None, None, "none", BF16, y[at], y[at].cpu(), (dx[at], None, None), BF16)
    torch.testing.assert_close(y[::1009, 0].float(), x[::1009].float() @ w[0].float(), rtol=2.0 ** -7, atol=2.0 ** -16)
