"""The norms around a residual block on the GPU against plain float64 computations.

Tolerances are bounds, not fits: `unit(type)` is the largest relative error of
one rounding to a type; a float32 sum of n terms held in lanes is off by at most
(n / 16 + 32) roundings of its terms' magnitudes; each check adds up what the
formula's steps can do.
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


def norm(v, e_v, layer, eps):
    """(unit row, 1 / deviation, error bound of the unit row) for a row v known to e_v."""
    d = v.shape[1]
    mu = v.mean(1, keepdim=True) if layer else torch.zeros(len(v), 1, dtype=torch.float64)
    c = v - mu
    r = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    n = c * r
    top = e_v.amax(1, keepdim=True) + sums(d) * v.abs().amax(1, keepdim=True) * (1 if layer else 0)
    # the centred value, then the deviation (its sum, and what the centred values' errors do to it), then two roundings
    e_c = top + EPS * c.abs()
    e = r * e_c + n.abs() * (2 * sums(d) + 8 * EPS + r * top)
    return n, r, e


def back(dy, e_dy, w, n, e_n, r, e_r, layer):
    """(gradient through norm(v) w + b, its error bound)."""
    d = n.shape[1]
    g, e_g = dy * w, e_dy * w.abs() + 2 * EPS * (dy * w).abs()
    c1 = g.mean(1, keepdim=True) if layer else torch.zeros_like(r)
    c2 = (g * n).mean(1, keepdim=True)
    G, E = g.abs().mean(1, keepdim=True), e_g.mean(1, keepdim=True)
    e_c1 = (E + sums(d) * G) if layer else torch.zeros_like(r)
    e_c2 = (e_g * n.abs() + g.abs() * e_n).mean(1, keepdim=True) + sums(d) * (g * n).abs().mean(1, keepdim=True)
    t = g - c1 - n * c2
    size = g.abs() + c1.abs() + (n * c2).abs()
    e = r * (e_g + e_c1 + e_n * c2.abs() + n.abs() * e_c2 + 6 * EPS * size) + e_r * r * size
    return r * t, e


def check(c, got, dt, pt, grads=None):
    layer, post, pre, eps, s = c["norm"] == "layer", c["post"], c["pre"], c["eps"], c["scale"]
    D = {k: None if c.get(k) is None else c[k].double() for k in ("x", "f", "gate", "pw", "pb", "w", "b", "dh", "dy")}
    x, f = D["x"], D["f"]
    d, rows = x.shape[1], x.shape[0]
    one, zero = torch.ones(d, dtype=torch.float64), torch.zeros(d, dtype=torch.float64)
    pw, pb, w, b = (zero if D[k] is None and k in ("pb", "b") else one if D[k] is None else D[k] for k in ("pw", "pb", "w", "b"))
    g = one if D["gate"] is None else D["gate"]
    Z = torch.zeros_like(x)
    fn, fr, e_fn = norm(f, Z, layer, eps) if post else (f, torch.ones(rows, 1, dtype=torch.float64), Z)
    e_fr = 2 * sums(d) + 8 * EPS if post else 0.0
    u = fn * pw + pb if post else f
    e_u = e_fn * pw.abs() + 3 * EPS * (u.abs() + (fn * pw).abs()) if post else Z
    h = s * x + g * u
    e_h = g.abs() * e_u + 3 * EPS * ((s * x).abs() + (g * u).abs())
    y = None
    if pre:
        hn, hr, e_hn = norm(h, e_h, layer, eps)
        e_hr = 2 * sums(d) + 8 * EPS + hr * (e_h.amax(1, keepdim=True) + sums(d) * h.abs().amax(1, keepdim=True))
        y = hn * w + b
        e_y = e_hn * w.abs() + 3 * EPS * (y.abs() + (hn * w).abs())
    if got is not None:
        within(got[0], h, 1.01 * (unit(dt) * h.abs() + e_h) + tiny(dt), "h")
        if pre:
            within(got[1], y, 1.01 * (unit(dt) * y.abs() + e_y) + tiny(dt), "y")
        else:
            assert got[1] is None
    if grads is None:
        return
    T = Z if D["dh"] is None else D["dh"]
    e_T = EPS * T.abs()
    ok = 1.01
    col = lambda v, e: (v.sum(0), e.sum(0) + sums(rows) * v.abs().sum(0))  # noqa: E731

    def vector(name, t, v, e):
        if t is not None:
            want, err = col(v, e)
            within(t, want, ok * (unit(pt) * want.abs() + err) + tiny(pt), name)

    if D["dy"] is not None:
        dy = D["dy"]
        t, e = back(dy, Z, w, hn, e_hn, hr, e_hr, layer)
        T, e_T = T + t, e_T + e + 2 * EPS * (T.abs() + t.abs())
        vector("dw", grads.dweight, dy * hn, dy.abs() * e_hn + EPS * (dy * hn).abs())
        vector("db", grads.dbias, dy, Z)
    within(grads.dx, s * T, ok * (unit(dt) * (s * T).abs() + abs(s) * e_T + EPS * (s * T).abs()) + tiny(dt), "dx")
    dg, e_dg = T * u, e_T * u.abs() + T.abs() * e_u + 2 * EPS * (T * u).abs()
    if grads.dgate is not None:
        if grads.dgate.shape == x.shape:
            within(grads.dgate, dg, ok * (unit(dt) * dg.abs() + e_dg) + tiny(dt), "dgate")
        else:
            vector("dgate", grads.dgate, dg, e_dg)
    du, e_du = T * g, e_T * g.abs() + EPS * (T * g).abs()
    if post:
        vector("dpw", grads.dpost_weight, du * fn, e_du * fn.abs() + du.abs() * e_fn + EPS * (du * fn).abs())
        vector("dpb", grads.dpost_bias, du, e_du)
        du, e_du = back(du, e_du, pw, fn, e_fn, fr, e_fr, layer)
    within(grads.df, du, ok * (unit(dt) * (du.abs() + e_du) + e_du) + tiny(dt), "df")


def case(rows, d, dt, pt, seed, post=True, pre=True, gate="features", norm="layer", scale=0.75, params=True, gap=0, eps=1e-5):
    g = gen(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    rowsof = lambda m=1.0, o=0.0: (r(rows, d + gap) * m + o).to(dt)[:, :d]  # noqa: E731
    vec = lambda o, m: (o + m * r(d)).to(pt)  # noqa: E731
    c = dict(norm=norm, post=post, pre=pre, eps=eps, scale=scale, x=rowsof(2, 0.5), f=rowsof(1.5, -0.3), dh=rowsof(), dy=rowsof() if pre else None)
    c.update(gate=None if gate is None else vec(0.5, 0.3) if gate == "features" else torch.sigmoid(r(rows, d)).to(dt))
    if params:
        c.update(w=vec(1, 0.3) if pre else None, b=vec(0, 0.3) if pre else None, pw=vec(1, 0.3) if post else None,
                 pb=vec(0, 0.3) if post else None)
    return c


def cu(t):
    if t is None or not isinstance(t, torch.Tensor):
        return t
    if t.dim() == 2 and t.shape[0] > 1 and t.stride(0) != t.shape[1]:
        wide = torch.full((t.shape[0], t.stride(0)), 7.0, dtype=t.dtype, device="cuda")
        wide[:, :t.shape[1]] = t.cuda()
        return wide[:, :t.shape[1]]
    return t.cuda()


def call(c, **kw):
    k = {n: cu(v) for n, v in c.items()}
    args = dict(scale=c["scale"], post=c["post"], post_weight=k.get("pw"), post_bias=k.get("pb"), pre=c["pre"], weight=k.get("w"),
                bias=k.get("b"), norm=c["norm"], **kw)
    h, y, stats = boa.block_norm_forward(k["x"], k["f"], k["gate"], eps=c["eps"], **args)
    r = boa.block_norm_backward(k["dh"], k["dy"], k["x"], k["f"], stats, k["gate"], **args)
    return (h, y, stats), r


def both(*a, **kw):
    c = case(*a, **kw)
    got, r = call(c)
    dt, pt = a[2], a[3]
    assert got[0].dtype == r.dx.dtype == r.df.dtype == dt
    check(c, got, dt, pt, r)
    return c, got, r


TYPES = [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)]


@pytest.mark.parametrize("dt,pt", TYPES)
@pytest.mark.parametrize("rows,d", [(1, 1), (1, 768), (3, 2), (5, 7), (2, 8), (5, 63), (7, 64), (4, 65), (9, 96), (33, 128), (17, 255),
                                    (6, 256), (8, 257), (19, 413), (64, 512), (5, 520), (30, 768), (3, 1000), (12, 1024),
                                    (5, 1025), (3, 1536), (4, 2048), (3, 2055), (3, 4095), (3, 4096), (2, 4097), (3, 8192), (5, 8191), (2, 8193), (2, 9000)])
def test_block_norm(rows, d, dt, pt):
    n = rows + d
    both(rows, d, dt, pt, n, gate=("features", "rows", None)[n % 3], norm=("layer", "rms")[n % 2], post=n % 5 != 0)


@pytest.mark.parametrize("dt,pt", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("gate", [None, "features", "rows"])
@pytest.mark.parametrize("post,pre", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("d", [200, 4500, 8200])
def test_every_form(d, post, pre, gate, kind, dt, pt):
    both(13, d, dt, pt, 3, post=post, pre=pre, gate=gate, norm=kind)
    both(13, d, dt, pt, 4, post=post, pre=pre, gate=gate, norm=kind, params=False)


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("rows,d", [(9000, 96), (3001, 413), (4200, 1024), (1100, 2048), (600, 8192), (70, 8200)])
def test_many_rows(rows, d, dt):
    c, got, r = both(rows, d, dt, dt, d)
    again, r2 = call(c)
    for a, b in zip((*got, *vars(r).values()), (*again, *vars(r2).values())):
        assert torch.equal(a, b)


@pytest.mark.parametrize("gate", ["features", "rows"])
@pytest.mark.parametrize("gap", [8, 3])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_strided_rows(gap, gate, dt):
    both(37, 200, dt, dt, 5, gap=gap, gate=gate)
    both(37, 5, dt, dt, 6, gap=gap, gate=gate)


@pytest.mark.parametrize("d", [96, 5000, 9000])
def test_one_of_the_gradients(d):
    c = case(21, d, F32, F32, 8)
    check(c | {"dh": None}, None, F32, F32, call(c | {"dh": None})[1])
    r = call(c | {"dy": None})[1]
    # without dy nothing comes back through the second norm
    assert torch.equal(r.dweight, torch.zeros_like(r.dweight)) and torch.equal(r.dbias, torch.zeros_like(r.dbias))
    T = c["dh"].double()
    within(r.dx, 0.75 * T, 4 * EPS * T.abs(), "dx")
    k = {n: cu(v) for n, v in c.items()}
    _, _, stats = boa.block_norm_forward(k["x"], k["f"], k["gate"], post=True, weight=k["w"])
    r = boa.block_norm_backward(k["dh"], k["dy"], k["x"], k["f"], stats, k["gate"], post=True, weight=k["w"], need_gate=False,
                                need_params=False)
    assert r.dgate is r.dweight is r.dbias is r.dpost_weight is None and r.dx is not None


def test_leading_dimensions_and_no_rows():
    c = case(24, 96, F32, F32, 3, gate="rows")
    k = {n: cu(v) for n, v in c.items()}
    shape = (2, 3, 4, 96)
    h, y, stats = boa.block_norm_forward(k["x"].reshape(shape), k["f"].reshape(shape), k["gate"].reshape(shape), 0.75, True, k["pw"],
                                         k["pb"], True, k["w"], k["b"])
    assert h.shape == y.shape == shape
    check(c, (h.reshape(24, 96), y.reshape(24, 96)), F32, F32)
    x = torch.empty(0, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    h, y, stats = boa.block_norm_forward(x, x, w, post=True, post_weight=w, weight=w, bias=w)
    r = boa.block_norm_backward(h, y, x, x, stats, w, post=True, post_weight=w, weight=w, bias=w)
    assert h.shape == r.df.shape == (0, 64)
    for t in (r.dgate, r.dweight, r.dbias, r.dpost_weight):
        assert torch.equal(t, torch.zeros_like(w))
    one = boa.block_norm_forward(k["x"][0], k["f"][0], k["pw"], 1.0)   # a row without leading dimensions, and a shared gate
    assert one[0].shape == (96,)
    within(one[0], c["x"][0].double() + c["pw"].double() * c["f"][0].double(), torch.full((96,), 1e-5).double(), "h")


def test_constant_rows_and_nan():
    x = torch.full((3, 96), 7.25, device="cuda")
    h, y, stats = boa.block_norm_forward(x, torch.zeros_like(x))
    assert torch.equal(y, torch.zeros_like(y)) and torch.equal(h, x) and torch.equal(stats[2], x[:, 0])
    for d in (300, 4500):
        c = case(6, d, F32, F32, 2)
        c["f"][2, 17] = math.nan
        c["x"][4, 3] = math.inf
        c["dh"][1, 0] = math.nan
        got, r = call(c)
        rows = lambda t: (~torch.isfinite(t)).any(1).cpu().nonzero().flatten().tolist()  # noqa: E731
        assert rows(got[0]) == rows(got[1]) == [2, 4]
        assert rows(r.df) == [1, 2, 4]


def test_autograd():
    c = case(40, 72, F32, F32, 12)
    names = ("x", "f", "gate", "pw", "pb", "w", "b")
    leaves = {n: c[n].cuda().requires_grad_() for n in names}
    kw = dict(scale=0.75, post=True, post_weight=leaves["pw"], post_bias=leaves["pb"], weight=leaves["w"], bias=leaves["b"])
    h, y = boa.block_norm(leaves["x"], leaves["f"], leaves["gate"], **kw)
    torch.autograd.backward([h, y], [c["dh"].cuda(), c["dy"].cuda()])
    r = boa.ops.BlockNormGrads(leaves["x"].grad, leaves["f"].grad, leaves["gate"].grad, leaves["pw"].grad, leaves["pb"].grad,
                               leaves["w"].grad, leaves["b"].grad)
    check(c, (h, y), F32, F32, r)
    # only the residual stream is used on
    x = c["x"].cuda().requires_grad_()
    h, y = boa.block_norm(x, c["f"].cuda(), pre=False)
    assert y is None
    h.sum().backward()
    assert torch.equal(x.grad, torch.ones_like(x))


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_gradient_against_differences(kind):
    c = case(9, 40, F32, F32, 31, norm=kind)
    _, r = call(c)
    layer = kind == "layer"
    names = ("x", "f", "gate", "pw", "pb", "w", "b")
    D = {n: c[n].double() for n in names}

    def loss(v):
        z = torch.zeros_like(v["x"])
        u = norm(v["f"], z, layer, 1e-5)[0] * v["pw"] + v["pb"]
        h = 0.75 * v["x"] + v["gate"] * u
        y = norm(h, z, layer, 1e-5)[0] * v["w"] + v["b"]
        return float((h * c["dh"].double() + y * c["dy"].double()).sum())

    grads = dict(x=r.dx, f=r.df, gate=r.dgate, pw=r.dpost_weight, pb=r.dpost_bias, w=r.dweight, b=r.dbias)
    g, step = gen(5), 1e-4
    for n in names:
        t = torch.randn(D[n].shape, generator=g, dtype=torch.float64)
        want = (loss(D | {n: D[n] + step * t}) - loss(D | {n: D[n] - step * t})) / (2 * step)
        terms = grads[n].double().cpu() * t
        assert abs(float(terms.sum()) - want) <= 1e-5 * float(terms.abs().sum()), n


def test_another_stream_and_captured():
    c = case(150, 300, BF16, BF16, 6)
    want, wr = call(c)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    k = {n: cu(v) for n, v in c.items()}
    kw = dict(scale=c["scale"], post=True, post_weight=k["pw"], post_bias=k["pb"], weight=k["w"], bias=k["b"])
    torch.cuda.synchronize()
    got = boa.block_norm_forward(k["x"], k["f"], k["gate"], stream=s, **kw)
    r = boa.block_norm_backward(k["dh"], k["dy"], k["x"], k["f"], got[2], k["gate"], stream=s, **kw)
    s.synchronize()
    for a, b in zip((*want, *vars(wr).values()), (*got, *vars(r).values())):
        assert torch.equal(a, b)

    def step():
        h, y, stats = boa.block_norm_forward(k["x"], k["f"], k["gate"], **kw)
        return (h, y, *vars(boa.block_norm_backward(h, y, k["x"], k["f"], stats, k["gate"], **kw)).values())

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for i in range(3):
        k["x"].copy_(torch.randn(150, 300, generator=gen(i)).bfloat16())
        g.replay()
        mine = [t.clone() for t in out]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(mine, step()))


def test_more_rows_than_a_launch_takes():
    # launches of 2^23 rows; offsets pass 2^32 bytes
    rows, d = (1 << 23) + 77, 264
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.randn(rows, d, device="cuda", generator=g).bfloat16()
    f = torch.randn(rows, d, device="cuda", generator=g).bfloat16()
    h, y, stats = boa.block_norm_forward(x, f, post=True)
    r = boa.block_norm_backward(h, y, x, f, stats, post=True)
    for at in (slice(0, 50), slice((1 << 23) - 20, (1 << 23) + 30), slice(rows - 50, rows)):
        c = dict(norm="layer", post=True, pre=True, eps=1e-5, scale=1.0, x=x[at].cpu(), f=f[at].cpu(), dh=h[at].cpu(), dy=y[at].cpu())
        part = boa.ops.BlockNormGrads(r.dx[at], r.df[at])
        check(c, (h[at], y[at]), BF16, BF16, part)
