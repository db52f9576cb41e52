"""Query-tower operators on the GPU against plain float64 computations.

Tolerances are bounds, not fits: `unit(type)` is the largest relative error of
one rounding to a type; a float32 sum of n terms held in lanes or matrix
instructions is off by at most (n / 16 + 32) roundings of its terms'
magnitudes; each test adds up what the formula's steps can do.
"""
import math

import pytest
import torch

import paper_2609_16175_amd as boa

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = 2.0 ** -24


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


# ---------------------------------------------------------------------------
# layer norm

def norm_case(rows, d, dt, pt, seed=0, gap=0, offset=0.5):
    g = gen(seed)
    wide = (torch.randn(rows, d + gap, generator=g) * 2 + offset).to(dt)
    dy = (torch.randn(rows, d + gap, generator=g)).to(dt)
    w = (1 + 0.3 * torch.randn(d, generator=g)).to(pt)
    b = (0.3 * torch.randn(d, generator=g)).to(pt)
    return wide, dy, w, b


def norm_plain(x, dy, w, b, eps):
    x, dy = x.double(), dy.double()
    w = torch.ones(x.shape[-1], dtype=torch.float64) if w is None else w.double()
    mu = x.mean(1, keepdim=True)
    c = x - mu
    r = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    xh = c * r
    y = xh * w + (0 if b is None else b.double())
    g = dy * w
    dx = r * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dict(y=y, dx=dx, dw=(dy * xh).sum(0), db=dy.sum(0), r=r, xh=xh, g=g, x=x, dy=dy, w=w, mu=mu)


def norm_check(x, dy, w, b, eps, got, dt, pt):
    p = norm_plain(x, dy, w, b, eps)
    d, rows = x.shape[1], x.shape[0]
    y, dx, dw, db = got
    # xh: the mean's error over the row's magnitude, then two roundings and the variance's sum
    e_xh = p["r"] * sums(d) * p["x"].abs().amax(1, keepdim=True) + p["xh"].abs() * (2 * sums(d) + 8 * EPS)
    e_y = e_xh * p["w"].abs() + 4 * EPS * p["y"].abs().amax(1, keepdim=True)
    within(y, p["y"], 1.01 * (unit(dt) * p["y"].abs() + e_y) + tiny(dt), "y")
    G = p["g"].abs().mean(1, keepdim=True)
    X = p["xh"].abs().amax(1, keepdim=True)
    GX = (p["g"] * p["xh"]).abs().mean(1, keepdim=True)
    e_in = e_xh.amax(1, keepdim=True)
    e_dx = p["r"] * ((4 * sums(d) + 8 * EPS) * (p["g"].abs() + G + X * GX) + e_in * (GX + X * G) * 2)
    within(dx, p["dx"], 1.01 * (unit(dt) * p["dx"].abs() + e_dx) + tiny(dt), "dx")
    e_dw = (p["dy"].abs() * (e_xh + sums(rows) * p["xh"].abs())).sum(0)
    within(dw, p["dw"], 1.01 * (unit(pt) * p["dw"].abs() + e_dw) + tiny(pt), "dw")
    within(db, p["db"], 1.01 * (unit(pt) * p["db"].abs() + sums(rows) * p["dy"].abs().sum(0)) + tiny(pt), "db")


@pytest.mark.parametrize("dt,pt", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)])
@pytest.mark.parametrize("rows,d", [(1, 1), (1, 768), (3, 2), (5, 63), (7, 64), (4, 65), (9, 96), (33, 128), (17, 255),
                                    (6, 256), (8, 257), (19, 413), (64, 512), (5, 520), (130, 768), (3, 1000), (12, 1024),
                                    (5, 1025), (3, 1536), (4, 2048), (3, 4096), (2, 4097), (2, 8192), (3, 8200), (2, 12345)])
def test_layer_norm(rows, d, dt, pt):
    x, dy, w, b = norm_case(rows, d, dt, pt, seed=rows * 10007 + d)
    xc, dyc = x.cuda(), dy.cuda()
    y, mean, rstd = boa.layer_norm_forward(xc, w.cuda(), b.cuda(), 1e-5)
    dx, dw, db = boa.layer_norm_backward(dyc, xc, w.cuda(), mean, rstd)
    assert y.dtype == dx.dtype == dt and dw.dtype == db.dtype == pt
    norm_check(x, dy, w, b, 1e-5, (y, dx, dw, db), dt, pt)


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("rows,d", [(2500, 96), (9000, 128), (3001, 413), (1200, 1024), (1100, 2048)])
def test_layer_norm_many_rows(rows, d, dt):
    x, dy, w, b = norm_case(rows, d, dt, dt, seed=d)
    xc = x.cuda()
    y, mean, rstd = boa.layer_norm_forward(xc, w.cuda(), b.cuda(), 1e-5)
    got = boa.layer_norm_backward(dy.cuda(), xc, w.cuda(), mean, rstd)
    norm_check(x, dy, w, b, 1e-5, (y, *got), dt, dt)
    again = boa.layer_norm_backward(dy.cuda(), xc, w.cuda(), mean, rstd)
    assert all(torch.equal(a, c) for a, c in zip(got, again))


@pytest.mark.parametrize("gap,start", [(8, 0), (3, 0), (8, 8), (5, 1)])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_layer_norm_strided_rows(gap, start, dt):
    wide, dyw, w, b = norm_case(37, 200, dt, dt, seed=5, gap=gap + start)
    x, dy = wide[:, start:start + 200], dyw[:, start:start + 200]
    xc, dyc = wide.cuda()[:, start:start + 200], dyw.cuda()[:, start:start + 200]
    assert not xc.is_contiguous()
    y, mean, rstd = boa.layer_norm_forward(xc, w.cuda(), b.cuda())
    got = boa.layer_norm_backward(dyc, xc, w.cuda(), mean, rstd)
    norm_check(x, dy, w, b, 1e-5, (y, *got), dt, dt)


def test_layer_norm_without_parameters_and_leading_dimensions():
    x, dy, _, _ = norm_case(24, 96, F32, F32, seed=3)
    xc = x.cuda().reshape(2, 3, 4, 96)
    y, mean, rstd = boa.layer_norm_forward(xc)
    dx, dw, db = boa.layer_norm_backward(dy.cuda().reshape(xc.shape), xc, None, mean, rstd)
    assert y.shape == dx.shape == xc.shape
    norm_check(x, dy, None, None, 1e-5, (y.reshape(24, 96), dx.reshape(24, 96), dw, db), F32, F32)


def test_layer_norm_no_rows():
    x = torch.empty(0, 64, device="cuda")
    y, mean, rstd = boa.layer_norm_forward(x, torch.ones(64, device="cuda"))
    dx, dw, db = boa.layer_norm_backward(x, x, torch.ones(64, device="cuda"), mean, rstd)
    assert y.shape == dx.shape == (0, 64)
    assert torch.equal(dw, torch.zeros_like(dw)) and torch.equal(db, torch.zeros_like(db))


def test_layer_norm_large_mean_and_constant_rows():
    # the variance comes from x - mean: a mean 4096 times the spread costs its share of digits and no more
    x = torch.randn(8, 768, generator=gen(1)) + 4096
    y, _, _ = boa.layer_norm_forward(x.cuda())
    p = norm_plain(x, x, None, None, 1e-5)
    within(y, p["y"], p["r"] * sums(768) * 4100 + 1e-5, "y")
    c = torch.full((3, 96), 7.25)
    y, mean, rstd = boa.layer_norm_forward(c.cuda(), eps=1e-5)
    assert torch.equal(y.cpu(), torch.zeros(3, 96)) and torch.equal(mean.cpu(), torch.full((3,), 7.25))
    within(rstd, torch.full((3,), 1e-5, dtype=F32).double().rsqrt(), 4 * EPS * 317, "rstd")


def test_layer_norm_nan_stays_in_its_row():
    x = torch.randn(6, 300, generator=gen(2))
    x[2, 17] = math.nan
    x[4, 3] = math.inf
    y, _, _ = boa.layer_norm_forward(x.cuda())
    bad = torch.isnan(y).any(1).cpu()
    assert bad.tolist() == [False, False, True, False, True, False]


def test_layer_norm_autograd_and_differences():
    x, dy, w, b = norm_case(6, 40, F32, F32, seed=8)
    xs, ws, bs = (t.cuda().requires_grad_() for t in (x, w, b))
    y = boa.layer_norm(xs, ws, bs, 1e-5)
    (y * dy.cuda()).sum().backward()
    norm_check(x, dy, w, b, 1e-5, (y, xs.grad, ws.grad, bs.grad), F32, F32)

    def f(x, w, b):
        return float((boa.layer_norm_forward(x.cuda(), w.cuda(), b.cuda())[0].double() * dy.cuda().double()).sum())

    g = gen(9)
    for t, grad, at in ((x, xs.grad, 0), (w, ws.grad, 1), (b, bs.grad, 2)):
        v = torch.randn(t.shape, generator=g)
        h = 1e-2
        args = [[x, w, b], [x, w, b]]
        args[0][at], args[1][at] = t + h * v, t - h * v
        diff = (f(*args[0]) - f(*args[1])) / (2 * h)
        want = float((grad.cpu().double() * v.double()).sum())
        # central differences: h^2 of curvature, and the float32 values' error over h
        assert abs(diff - want) < 2e-2 * (1 + abs(want))


# ---------------------------------------------------------------------------
# softmax cross entropy

def xent_case(B, V, d, dt, seed=0, bias=True, ignored=0.2, out=0.05):
    g = gen(seed)
    pts = torch.randn(V, d, generator=g)
    pts = (pts / pts.norm(dim=1, keepdim=True)).to(dt)
    labels = torch.randint(V, (B,), generator=g)
    h = pts.float()[labels] + 0.7 * torch.randn(B, d, generator=g) / math.sqrt(d)
    h = h.to(dt)
    bm = None
    if bias:
        bm = 0.5 * torch.randn(V, generator=g)
        drop = torch.rand(V, generator=g) < out
        drop[labels] = False
        bm[drop] = -math.inf
    labels[torch.rand(B, generator=g) < ignored] = -1
    return h, pts, labels, bm


def xent_plain(h, pts, labels, bias, scale, reduction, dloss=None):
    h, c = h.double(), pts.double()
    l = scale * (h @ c.t()) + (0 if bias is None else bias.double())
    lse = torch.logsumexp(l, 1)
    valid = labels >= 0
    at = labels.clamp(min=0)
    rows = torch.arange(h.shape[0])
    loss = torch.where(valid, lse - l[rows, at], torch.zeros_like(lse))
    n = max(1, int(valid.sum())) if reduction == "mean" else 1
    g = valid.double() / n
    if dloss is not None:
        g = g * dloss.double()
    p = torch.exp(l - lse[:, None])
    q = p.clone()
    q[rows, at] -= 1
    q = q * g[:, None]
    total = loss if reduction == "none" else loss.sum() / n
    return dict(l=l, lse=lse, loss=total, rows=loss, p=p, q=q, g=g, dh=scale * q @ c, drows=scale * q.t() @ h, dbias=q.sum(0),
                h=h, c=c, valid=valid, n=n)


def xent_check(case, got, dt, scale, reduction, dloss=None, what=("dh", "drows", "dbias")):
    h, pts, labels, bias = case
    p = xent_plain(h, pts, labels, bias, scale, reduction, dloss)
    d, (B, V) = h.shape[1], p["l"].shape
    mag = scale * (p["h"].abs() @ p["c"].abs().t())
    e_l = sums(6 * d) * float(mag.max()) + 8 * EPS * float(p["l"][torch.isfinite(p["l"])].abs().max())
    e_lse = e_l + (sums(V) + 8 * EPS) + 4 * EPS * p["lse"].abs().max()
    e_rows = 2 * e_lse + 4 * EPS * p["rows"].abs()
    if reduction == "none":
        within(got.loss, p["loss"], e_rows, "loss")
    else:
        e = (e_rows * p["valid"]).sum() / p["n"] + sums(B) * p["rows"].abs().sum() / p["n"]
        within(got.loss, p["loss"], e, "loss")
    within(got.lse, p["lse"], e_lse + 4 * EPS * p["lse"].abs(), "lse")
    # relative error of a probability, and its rounding (three bf16 parts of float32 hold its 24 bits)
    e_p = 2 * e_lse + 16 * EPS
    u = unit(dt)
    e_q = p["p"] * p["g"].abs()[:, None] * (e_p + u + sums(6 * V + 6 * B))
    at = labels.clamp(min=0)
    rows = torch.arange(B)
    e_q[rows, at] = p["g"].abs() * (p["p"][rows, at] * e_p + 32 * EPS)
    full = p["q"].abs()
    if "dh" in what:
        e = scale * (e_q @ p["c"].abs() + sums(6 * V) * full @ p["c"].abs()) + u * p["dh"].abs()
        within(got.dh, p["dh"], 1.02 * e, "dh")
    if "drows" in what:
        e = scale * (e_q.t() @ p["h"].abs() + sums(6 * B) * full.t() @ p["h"].abs()) + u * p["drows"].abs()
        within(got.drows, p["drows"], 1.02 * e + 1e-42, "drows")
    if "dbias" in what and bias is not None:
        e_qb = p["p"] * p["g"].abs()[:, None] * (e_p + 8 * EPS)
        e_qb[rows, at] = p["g"].abs() * (p["p"][rows, at] * e_p + 8 * EPS)
        within(got.dbias, p["dbias"], 1.02 * (e_qb.sum(0) + sums(B) * full.sum(0)) + 1e-42, "dbias")


def xent_run(case, scale, reduction="mean", dloss=None, **kw):
    h, pts, labels, bias = (None if t is None else t.cuda() for t in case)
    return boa.softmax_xent_grad(h, pts, labels, bias, scale, reduction, dloss=dloss, bias_grad=bias is not None, **kw)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("B,V,d", [(1, 1, 1), (1, 7, 3), (2, 33, 16), (5, 255, 17), (31, 256, 32), (32, 257, 33),
                                   (33, 300, 48), (64, 1000, 64), (65, 511, 65), (100, 2000, 96), (127, 513, 127),
                                   (128, 1500, 128), (129, 1025, 129), (200, 3000, 130), (255, 777, 192), (257, 1024, 200),
                                   (300, 1300, 256), (70, 2100, 257), (40, 900, 768), (9, 400, 1024), (3, 300, 2050),
                                   (600, 5000, 100)])
def test_softmax_xent(B, V, d, dt):
    case = xent_case(B, V, d, dt, seed=B * 31 + V + d, bias=(B + d) % 2 == 1, ignored=0.2 if B > 2 else 0.0)
    got = xent_run(case, 8.0)
    assert got.dh.dtype == got.drows.dtype == dt
    xent_check(case, got, dt, 8.0, "mean")


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("reduction", ["none", "sum", "mean"])
@pytest.mark.parametrize("d", [64, 300])
def test_softmax_xent_reductions(reduction, dt, d):
    case = xent_case(50, 700, d, dt, seed=2)
    g = gen(4)
    dloss = torch.randn(50, generator=g) if reduction == "none" else torch.tensor(-1.75)
    got = xent_run(case, 6.0, reduction, dloss=dloss.cuda())
    xent_check(case, got, dt, 6.0, reduction, dloss=dloss)


@pytest.mark.parametrize("d", [96, 384])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_softmax_xent_pieces(dt, d):
    # more queries than one piece of the points' probabilities holds; every point repeats among the labels
    case = xent_case(2100, 40_000 if d == 96 else 36_000, d, dt, seed=6, ignored=0.01)
    case[2][500:900] = case[2][0]
    got = xent_run(case, 10.0)
    xent_check(case, got, dt, 10.0, "mean")
    again = xent_run(case, 10.0)
    assert all(torch.equal(getattr(got, k), getattr(again, k)) for k in ("loss", "lse", "dh", "drows", "dbias"))


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("d", [40, 320])
def test_softmax_xent_equal_labels(dt, d):
    case = xent_case(300, 500, d, dt, seed=7, ignored=0.0)
    case[2][:] = 123
    case[3][123] = 0.25
    got = xent_run(case, 5.0)
    xent_check(case, got, dt, 5.0, "mean")


@pytest.mark.parametrize("dt", [F32, BF16])
def test_softmax_xent_some_gradients(dt):
    case = xent_case(80, 900, 112, dt, seed=11)
    whole = xent_run(case, 4.0)
    h, pts, labels, bias = (t.cuda() for t in case)
    for a, b, c in ((True, False, False), (False, True, False), (False, False, True), (False, False, False)):
        r = boa.softmax_xent_grad(h, pts, labels, bias, 4.0, h_grad=a, rows_grad=b, bias_grad=c)
        assert (r.dh is not None, r.drows is not None, r.dbias is not None) == (a, b, c)
        for k in ("loss", "dh", "drows", "dbias"):
            one = getattr(r, k)
            assert one is None or torch.equal(one, getattr(whole, k))
    assert torch.equal(boa.softmax_xent(h, pts, labels, bias, 4.0), whole.loss)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("d", [32, 80, 288])
def test_softmax_xent_empty_rows(dt, d):
    h, pts, labels, bias = xent_case(40, 300, d, dt, seed=12, ignored=0.0)
    # every query left out: loss 0, gradients 0
    r = xent_run((h, pts, torch.full_like(labels, -5), bias), 3.0)
    assert float(r.loss) == 0 and all(not t.any() for t in (r.dh, r.drows, r.dbias))
    # every point left out: loss +inf, gradients 0, no NaN
    r = xent_run((h, pts, labels, torch.full_like(bias, -math.inf)), 3.0, "none")
    assert torch.isposinf(r.loss).all() and torch.isneginf(r.lse).all()
    assert all(not t.any() for t in (r.dh, r.drows, r.dbias))
    # the lowest finite bias is a number like any other
    low = torch.full_like(bias, torch.finfo(F32).min)
    r = xent_run((h, pts, labels, low), 3.0, "none")
    assert torch.isfinite(r.loss).all() and torch.isfinite(r.dh.float()).all() and torch.isfinite(r.drows.float()).all()
    # a label that is no point: NaN loss, nothing else touched
    bad = labels.clone()
    bad[7] = 300
    r = xent_run((h, pts, bad, bias), 3.0, "none")
    assert torch.isnan(r.loss[7]) and torch.isfinite(r.loss[:7]).all() and torch.isfinite(r.loss[8:]).all()
    assert not r.dh[7].any() and torch.isfinite(r.drows.float()).all()
    # a label whose point is left out: loss +inf, the other entries as ever
    out = bias.clone()
    out[labels[3]] = -math.inf
    r = xent_run((h, pts, labels, out), 3.0, "none")
    assert torch.isposinf(r.loss[3]) and torch.isfinite(r.dh.float()).all()


@pytest.mark.parametrize("d", [64, 272])
def test_softmax_xent_infinities_and_nan(d):
    h, pts, labels, bias = xent_case(40, 300, d, BF16, seed=13, ignored=0.0)
    labels[:] = torch.arange(40) + 10
    bias = torch.zeros(300)
    # a query of infinities or NaN is its own affair
    h2 = h.clone()
    h2[5, 3] = math.nan
    r = xent_run((h2, pts, labels, bias), 3.0, "none")
    assert torch.isnan(r.loss[5])
    keep = [i for i in range(40) if i != 5]
    clean = xent_run((h, pts, labels, bias), 3.0, "none")
    assert torch.equal(r.loss[keep], clean.loss[keep]) and torch.equal(r.dh[keep], clean.dh[keep])
    # left out, it touches neither losses nor the points
    labels2 = labels.clone()
    labels2[5] = -1
    r = xent_run((h2, pts, labels2, bias), 3.0, "none")
    assert float(r.loss[5]) == 0 and torch.isfinite(r.dh[keep].float()).all()


def test_softmax_xent_no_queries():
    h = torch.empty(0, 48, device="cuda")
    pts = torch.randn(100, 48, device="cuda")
    lab = torch.empty(0, dtype=torch.int64, device="cuda")
    r = boa.softmax_xent_grad(h, pts, lab, torch.zeros(100, device="cuda"), bias_grad=True)
    assert float(r.loss) == 0 and not r.drows.any() and not r.dbias.any() and r.dh.shape == (0, 48)
    assert boa.softmax_xent(h, pts, lab, reduction="none").shape == (0,)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("gap,start", [(8, 0), (8, 8), (3, 1)])
def test_softmax_xent_strides(dt, gap, start):
    h, pts, labels, bias = xent_case(50, 600, 96, dt, seed=14)
    def wide(t):
        w = torch.full((t.shape[0], t.shape[1] + gap + start), math.nan, dtype=dt, device="cuda")
        w[:, start:start + t.shape[1]] = t.cuda()
        return w[:, start:start + t.shape[1]]
    r = boa.softmax_xent_grad(wide(h), wide(pts), labels.cuda(), bias.cuda(), 4.0, bias_grad=True)
    xent_check((h, pts, labels, bias), r, dt, 4.0, "mean")


def test_softmax_xent_confident_queries_keep_their_digits():
    # probabilities of the labels near 1: the gradient is (p - 1) times its point, small and exact
    h, pts, labels, _ = xent_case(64, 400, 64, BF16, seed=15, bias=False, ignored=0.0)
    h = pts[labels].clone()
    case = (h, pts, labels, None)
    got = boa.softmax_xent_grad(h.cuda(), pts.cuda(), labels.cuda(), scale=16.0)
    xent_check(case, got, BF16, 16.0, "mean")


@pytest.mark.parametrize("reduction", ["none", "mean"])
def test_softmax_xent_autograd_and_differences(reduction):
    h, pts, labels, bias = xent_case(12, 90, 24, F32, seed=16, out=0.0)
    hs, ps, bs = (t.cuda().requires_grad_() for t in (h, pts, bias))
    wts = torch.rand(12, generator=gen(3)) + 0.5
    loss = boa.softmax_xent(hs, ps, labels.cuda(), bs, 5.0, reduction)
    top = (loss * wts.cuda()).sum() if reduction == "none" else 3.0 * loss
    top.backward()
    dloss = wts if reduction == "none" else torch.tensor(3.0)
    got = boa.ops.XentResult(loss, boa.softmax_xent_grad(h.cuda(), pts.cuda(), labels.cuda(), bias.cuda(), 5.0).lse, hs.grad,
                             ps.grad, bs.grad)
    xent_check((h, pts, labels, bias), got, F32, 5.0, reduction, dloss=dloss)

    def f(h, p, b):
        x = boa.softmax_xent(h.cuda(), p.cuda(), labels.cuda(), b.cuda(), 5.0, "none").double().cpu()
        n = max(1, int((labels >= 0).sum()))
        return float((x * wts.double()).sum()) if reduction == "none" else 3.0 * float(x.sum()) / n

    g = gen(17)
    for at, (t, grad) in enumerate(((h, hs.grad), (pts, ps.grad), (bias, bs.grad))):
        v = torch.randn(t.shape, generator=g)
        step = 1e-2 / float(v.norm())
        a, b = [h, pts, bias], [h, pts, bias]
        a[at], b[at] = t + step * v, t - step * v
        diff = (f(*a) - f(*b)) / (2 * step)
        want = float((grad.cpu().double() * v.double()).sum())
        # losses of about 60 in all with 1e-6 of error each side, over 2e-2 / |v|; and the step's square
        assert abs(diff - want) < 2e-3 * float(v.norm()) + 1e-3 * abs(want)


def test_softmax_xent_offsets_past_32_bits():
    V, d, B = 2_900_000, 768, 3
    pts = torch.empty(V, d, dtype=BF16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))
    labels = torch.tensor([V - 1, 5, V - 70_000], device="cuda")
    h = (0.02 * pts[labels].float()).to(BF16)
    r = boa.softmax_xent_grad(h, pts, labels, reduction="none", rows_grad=True)
    l = torch.cat([h.double() @ c.double().t() for c in pts.split(100_000)], 1)
    lse = torch.logsumexp(l, 1)
    want = lse - l[torch.arange(B, device="cuda"), labels]
    assert (r.loss.double() - want).abs().max() < 1e-4
    p = torch.exp(l - lse[:, None])
    for v in (V - 1, V - 70_000, 5, V - 2):
        q = p[:, v] - (labels == v).double()
        row = q @ h.double()
        bound = ((p[:, v] * 2.0 ** -8 + 1e-4) @ h.double().abs()) + 2.0 ** -8 * row.abs()
        assert ((r.drows[v].double() - row).abs() <= bound).all()


# ---------------------------------------------------------------------------
# products with 4-bit rows

def rows4_case(M, N, K, group, dt, sdt, offsets, seed=0):
    g = gen(seed)
    G = -(-K // group)
    q = torch.randint(16, (N, K), generator=g, dtype=torch.uint8)
    even = q[:, 0::2]
    odd = torch.zeros_like(even)
    odd[:, :K // 2] = q[:, 1::2]
    if K % 2:
        odd[:, -1] = 13   # a nibble past the end, never read
    codes = even | (odd << 4)
    s = (0.02 * torch.rand(N, G, generator=g) + 0.001).to(sdt)
    o = (torch.randn(N, G, generator=g) * 0.1).to(sdt) if offsets else None
    x = torch.randn(M, K, generator=g).to(dt)
    return x, q, codes, s, o


def rows4_check(y, x, q, s, o, group, dt):
    K = q.shape[1]
    at = torch.arange(K) // group
    qd, sd, X = q.double(), s.double()[:, at], x.double()
    # with offsets the sum runs over s q and o apart, without over s (q - 8): the magnitudes that cancel
    w = sd * (qd - 8) if o is None else sd * qd + o.double()[:, at]
    mag = sd.abs() * (qd + 40) + (0 if o is None else o.double()[:, at].abs())
    want = X @ w.t()
    within(y, want, 1.01 * (unit(dt) * want.abs() + sums(3 * K) * (X.abs() @ mag.t())) + tiny(dt), "y")


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("offsets", [False, True])
@pytest.mark.parametrize("M,N,K,group", [(1, 1, 1, 1), (1, 3, 2, 2), (2, 5, 7, 3), (1, 17, 32, 32), (1, 16, 64, 32),
                                         (3, 33, 96, 32), (1, 100, 128, 128), (4, 31, 128, 64), (5, 65, 160, 32),
                                         (6, 200, 192, 96), (8, 129, 256, 256), (1, 768, 768, 32), (7, 500, 384, 128),
                                         (16, 300, 512, 64), (17, 70, 640, 64), (33, 40, 224, 32), (1, 50, 1000, 100),
                                         (2, 40, 1024, 1024), (1, 64, 4096, 128), (5, 48, 8192, 64), (1, 20, 9000, 1000)])
def test_matvec_4bit(M, N, K, group, dt, offsets):
    sdt = [F32, BF16, F16][(M + N) % 3]
    x, q, codes, s, o = rows4_case(M, N, K, group, dt, sdt, offsets, seed=N + K)
    y = boa.matvec_4bit(x.cuda(), codes.cuda(), s.cuda(), None if o is None else o.cuda(), group=group)
    assert y.dtype == dt and y.shape == (M, N)
    rows4_check(y, x, q, s, o, group, dt)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("M,N,K", [(1, 70_001, 128), (5, 40_003, 96), (3, 30_000, 768), (16, 9_001, 256)])
def test_matvec_4bit_many_rows(M, N, K, dt):
    x, q, codes, s, o = rows4_case(M, N, K, 32, dt, BF16, True, seed=1)
    y = boa.matvec_4bit(x.cuda(), codes.cuda(), s.cuda(), o.cuda())
    rows4_check(y, x, q, s, o, 32, dt)
    assert torch.equal(y, boa.matvec_4bit(x.cuda(), codes.cuda(), s.cuda(), o.cuda()))


@pytest.mark.parametrize("gap,start", [(16, 0), (16, 16), (3, 1)])
def test_matvec_4bit_strides(gap, start):
    x, q, codes, s, o = rows4_case(3, 130, 256, 64, BF16, F32, True, seed=2)
    def wide(t, by=1):
        w = torch.full((t.shape[0], t.shape[1] + gap + start), 77, dtype=t.dtype, device="cuda")
        w[:, start:start + t.shape[1]] = t.cuda()
        return w[:, start:start + t.shape[1]]
    rows4_check(boa.matvec_4bit(wide(x), wide(codes), wide(s), wide(o)), x, q, s, o, 64, BF16)
    # scales and offsets of different strides
    rows4_check(boa.matvec_4bit(wide(x), codes.cuda(), wide(s), o.cuda()), x, q, s, o, 64, BF16)


def test_matvec_4bit_vector_and_nothing():
    x, q, codes, s, o = rows4_case(1, 90, 128, 32, F32, F32, False, seed=3)
    y = boa.matvec_4bit(x[0].cuda(), codes.cuda(), s.cuda())
    assert y.shape == (90,)
    rows4_check(y[None], x, q, s, o, 32, F32)
    assert boa.matvec_4bit(x[:0].cuda(), codes.cuda(), s.cuda()).shape == (0, 90)
    assert boa.matvec_4bit(x.cuda(), codes[:0].cuda(), s[:0].cuda()).shape == (1, 0)


def test_matvec_4bit_wide_range():
    # float32 values whose parts span the type's range, and zeros
    x, q, codes, s, o = rows4_case(4, 60, 128, 32, F32, F32, True, seed=4)
    x[0] *= 1e30
    x[1] *= 1e-30
    x[2] = 0
    y = boa.matvec_4bit(x.cuda(), codes.cuda(), s.cuda(), o.cuda())
    rows4_check(y, x, q, s, o, 32, F32)
    assert not y[2].any()


def test_matvec_4bit_non_finite_vector_stays_alone():
    x, q, codes, s, o = rows4_case(3, 60, 128, 32, BF16, F32, True, seed=5)
    clean = boa.matvec_4bit(x.cuda(), codes.cuda(), s.cuda(), o.cuda())
    x[1, 5] = math.nan
    y = boa.matvec_4bit(x.cuda(), codes.cuda(), s.cuda(), o.cuda())
    assert torch.isnan(y[1]).all() and torch.equal(y[0], clean[0]) and torch.equal(y[2], clean[2])


def test_matvec_4bit_offsets_past_32_bits():
    N, K = 6_000_000, 1024   # 3 GB of codes
    codes = torch.randint(256, (N, K // 2), dtype=torch.uint8, device="cuda",
                          generator=torch.Generator("cuda").manual_seed(1))
    s = torch.full((N, 8), 0.01, device="cuda")
    x = torch.randn(1, K, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    y = boa.matvec_4bit(x, codes, s)
    for at in (0, N // 2, N - 50):
        c = codes[at:at + 50].cpu()
        q = torch.stack((c & 15, c >> 4), 2).reshape(50, K)
        rows4_check(y[:, at:at + 50], x.cpu(), q, s[at:at + 50].cpu(), None, 128, F32)


# ---------------------------------------------------------------------------
# streams, graphs, refusals

def test_other_stream_and_graph():
    h, pts, labels, bias = (t.cuda() for t in xent_case(60, 800, 64, BF16, seed=20))
    x, dy, w, b = (t.cuda() for t in norm_case(60, 64, BF16, BF16, seed=21))
    m, _, codes, s, o = rows4_case(2, 64, 64, 32, BF16, F32, True, seed=22)
    m, codes, s, o = (t.cuda() for t in (m, codes, s, o))

    def step(stream=None):
        y, mean, rstd = boa.layer_norm_forward(x, w, b, stream=stream)
        r = boa.softmax_xent_grad(h, pts, labels, bias, 4.0, bias_grad=True, stream=stream)
        g = boa.layer_norm_backward(dy, x, w, mean, rstd, stream=stream)
        return [y, r.loss, r.dh, r.drows, r.dbias, *g, boa.matvec_4bit(m, codes, s, o, stream=stream)]

    want = step()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = step(side)
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        for t in out:
            t.fill_(float("nan"))
        x.add_(0.125)
        h.mul_(1.25)
        m.mul_(0.5)
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(out, want)), k


def test_binding_refuses():
    dev = "cuda"
    x = torch.zeros(4, 32, device=dev)
    lab = torch.zeros(4, dtype=torch.int64, device=dev)
    with pytest.raises(boa.BoaError, match="float16"):
        boa.softmax_xent(x.half(), x.half(), lab)
    for bad in (lambda: boa.softmax_xent(x, x[:, :16], lab), lambda: boa.softmax_xent(x, x.bfloat16(), lab),
                lambda: boa.softmax_xent(x, x, lab[:3]), lambda: boa.softmax_xent(x, x, lab.int()),
                lambda: boa.softmax_xent(x, x, lab, bias=torch.zeros(3, device=dev)),
                lambda: boa.softmax_xent(x, x, lab, reduction="max"),
                lambda: boa.softmax_xent_grad(x, x, lab, bias_grad=True),
                lambda: boa.layer_norm(x, torch.ones(31, device=dev)),
                lambda: boa.layer_norm_backward(x[:2], x, None, x[:, 0], x[:, 0]),
                lambda: boa.matvec_4bit(x, torch.zeros(3, 15, dtype=torch.uint8, device=dev), torch.ones(3, 1, device=dev)),
                lambda: boa.matvec_4bit(x, torch.zeros(3, 16, dtype=torch.uint8, device=dev), torch.ones(3, 5, device=dev)),
                lambda: boa.matvec_4bit(x, torch.zeros(3, 16, dtype=torch.uint8, device=dev), torch.ones(3, 2, device=dev), group=8)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        boa.layer_norm(x.double())


# ---------------------------------------------------------------------------
# the operators together

def test_query_tower_example():
    from examples import query_tower
    from workloads import rows4
    r = query_tower.main(["--steps", "60", "--points", "3000"])
    assert r["last"] < 0.5 * r["first"] and r["found"] > 0.8 and r["found_4bit"] > 0.7
    # the served vectors are the tower's with the weights that the codes stand for
    w4 = rows4.dequantize(*rows4.quantize(r["W"], group=32)).double()
    w, b = (t.detach().double() for t in r["norm"])
    x = r["x"].double()
    c = x - x.mean(1, keepdim=True)
    y = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * w + b
    err = (r["served"].double() - y @ w4.t()).abs()
    assert (err <= 1e-5 * (y.abs() @ w4.abs().t()) + 1e-5).all()
