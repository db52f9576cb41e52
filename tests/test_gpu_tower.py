"""The operators of a query tower together, as a training step and a server
call them, on the GPU against plain float64 computations.

Each operator is checked on the tensors that it got from the one before it, with
the bounds of its own tests. The gradient of a whole tower is checked against
differences.
"""
import math

import pytest
import torch

import paper_2609_16175_amd as boa
import test_gpu_block_norm as blocks
import test_gpu_linear as linears
import test_gpu_orth as updates

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def parameters(d, wide, out, dt, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    p = dict(nw=1 + 0.2 * r(d), nb=0.2 * r(d), U0=r(wide, d) / d ** 0.5, u0=0.2 * r(wide), V0=r(d, wide) / wide ** 0.5, v0=0.2 * r(d),
             gate=0.5 + 0.2 * r(d), pw=1 + 0.2 * r(d), pb=0.2 * r(d), w0=1 + 0.2 * r(d), b0=0.2 * r(d), U1=r(wide, d) / d ** 0.5,
             u1=0.2 * r(wide), V1=r(d, wide) / wide ** 0.5, w1=1 + 0.2 * r(d), b1=0.2 * r(d), W=r(out, d) / d ** 0.5)
    return {k: v.to(dt).cuda() for k, v in p.items()}


def tower(x, p):
    """Every tensor of a tower of two blocks: one normed and gated, one added to the stream by its last product."""
    t = dict(x=x)
    t["y0"] = boa.layer_norm(x, p["nw"], p["nb"])
    t["a0"] = boa.linear(t["y0"], p["U0"], p["u0"], activation="gelu")
    t["f0"] = boa.linear(t["a0"], p["V0"], p["v0"])
    t["h1"], t["y1"] = boa.block_norm(x, t["f0"], p["gate"], post=True, post_weight=p["pw"], post_bias=p["pb"], weight=p["w0"],
                                      bias=p["b0"])
    t["a1"] = boa.linear(t["y1"], p["U1"], p["u1"], activation="silu")
    t["h2"] = boa.linear(t["a1"], p["V1"], residual=t["h1"])
    t["y2"] = boa.layer_norm(t["h2"], p["w1"], p["b1"])
    t["q"] = boa.linear(t["y2"], p["W"])
    return t


LAYERS = [("y0", "U0", "u0", None, "gelu", "a0"), ("a0", "V0", "v0", None, "none", "f0"), ("y1", "U1", "u1", None, "silu", "a1"),
          ("a1", "V1", None, "h1", "none", "h2"), ("y2", "W", None, None, "none", "q")]


def host(t):
    return None if t is None else t.detach().cpu()


def check(t, p, dt, grads=None):
    """grads: of every tensor by its name."""
    at = lambda n: None if n is None else host(t.get(n, p.get(n)))  # noqa: E731
    back = lambda n: None if n is None or grads is None else host(grads[n])  # noqa: E731
    for x, w, b, r, kind, y in LAYERS:
        linears.check(at(x), at(w), at(b), at(r), kind, dt, at(y), back(y), None if grads is None else (back(x), back(w), back(b)), dt)
    c = dict(norm="layer", post=True, pre=True, eps=1e-5, scale=1.0, x=at("x"), f=at("f0"), gate=at("gate"), pw=at("pw"), pb=at("pb"),
             w=at("w0"), b=at("b0"), dh=back("h1"), dy=back("y1"))
    blocks.check(c, (t["h1"], t["y1"]), dt, dt, None if grads is None else grads["block"])


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("M,d,wide,out,classes", [(70, 96, 384, 40, 300), (515, 200, 264, 64, 1000), (33, 33, 71, 17, 50)])
def test_training_step(M, d, wide, out, classes, dt):
    p = {k: v.requires_grad_() for k, v in parameters(d, wide, out, dt, M).items()}
    g = torch.Generator().manual_seed(M + 1)
    x = torch.randn(M, d, generator=g).to(dt).cuda()
    points = torch.randn(classes, out, generator=g).to(dt).cuda()
    labels = torch.randint(classes, (M,), generator=g).cuda()
    xs = x.clone().requires_grad_()   # of the first norm and of the block, whose shares are checked apart
    t = tower(x, p)
    mid = {k: v for k, v in t.items() if k != "x"}
    for v in mid.values():
        v.retain_grad()
    # the loss takes no float16; a large factor keeps gradients in float16 above its denormals
    q, points = (v.float() if dt == F16 else v for v in (t["q"], points))
    (boa.softmax_xent(q, points, labels, scale=0.5) * 64.0).backward()
    grads = {k: v.grad for k, v in (mid | p).items()}
    # the block's gradients with the one of x, which the tower's own x does not ask for
    k = {n: v.detach() for n, v in (t | p).items()}
    h, y = boa.block_norm(xs, k["f0"], k["gate"], post=True, post_weight=k["pw"], post_bias=k["pb"], weight=k["w0"], bias=k["b0"])
    torch.autograd.backward([h, y], [grads["h1"], grads["y1"]])
    grads["block"] = boa.ops.BlockNormGrads(xs.grad, grads["f0"], grads["gate"], grads["pw"], grads["pb"], grads["w0"], grads["b0"])
    check(t, p, dt, grads)
    for name in ("U0", "V0", "U1", "V1"):
        m = grads[name]
        updates.check_all(host(m), boa.orthogonalize(m), dt, [updates.CO] * 5)
    both = torch.stack([grads["U0"], grads["U1"]])
    assert torch.equal(boa.orthogonalize(both)[1], boa.orthogonalize(grads["U1"]))


@pytest.mark.parametrize("dt", [F32, BF16])
def test_serving(dt):
    # single states, a few of them, and many: each of the forms that a forward pass has
    p = parameters(160, 640, 96, dt, 5)
    x = torch.randn(90, 160, generator=torch.Generator().manual_seed(6)).to(dt).cuda()
    with torch.no_grad():
        for rows in (slice(0, 1), slice(41, 42), slice(3, 16), slice(0, 90)):
            check(tower(x[rows], p), p, dt)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_captured_step(dt):
    # forward, backward and the matrices' updates in one graph, replayed on new states
    p = parameters(96, 384, 40, dt, 8)
    x = torch.randn(130, 96, generator=torch.Generator().manual_seed(9)).to(dt).cuda()
    dq = torch.randn(130, 40, generator=torch.Generator().manual_seed(10)).to(dt).cuda()
    kw = dict(post=True, post_weight=p["pw"], post_bias=p["pb"], weight=p["w0"], bias=p["b0"])

    def step():
        y, mean, rstd = boa.layer_norm_forward(x, p["nw"], p["nb"])
        a, pre = boa.linear_forward(y, p["U0"], p["u0"], activation="gelu", keep=True)
        f, _ = boa.linear_forward(a, p["V0"], p["v0"])
        h, z, stats = boa.block_norm_forward(x, f, p["gate"], **kw)
        q, _ = boa.linear_forward(z, p["W"])
        dz, dW, _ = boa.linear_backward(dq, z, p["W"], need=(True, True, False))
        r = boa.block_norm_backward(None, dz, x, f, stats, p["gate"], **kw)
        da, dV, dv = boa.linear_backward(r.df, a, p["V0"])
        dy, dU, du = boa.linear_backward(da, y, p["U0"], pre, "gelu")
        dx, dnw, dnb = boa.layer_norm_backward(dy, x, p["nw"], mean, rstd)
        return q, dW, dV, dv, dU, du, dnw, dnb, dx, r.dx, r.dgate, boa.orthogonalize(dU), boa.orthogonalize(dV)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(3):
        x.copy_(torch.randn(130, 96, generator=torch.Generator().manual_seed(20 + k)).to(dt))
        graph.replay()
        got = [t.clone() for t in out]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, step()))


def plain_loss(v, x, points, labels, bias, scale, n_blocks):
    def norm(h, w, b):
        c = h - h.mean(1, keepdim=True)
        return c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * w + b

    h, y = x, norm(x, v["norm0"], v["norm1"])
    for i in range(n_blocks):
        b = {k: v[f"{k}{i}"] for k in ("up", "up_bias", "down", "down_bias", "gate", "weight", "bias")}
        f = linears.act(y @ b["up"].T + b["up_bias"], "gelu") @ b["down"].T + b["down_bias"]
        h = h + b["gate"] * f
        y = norm(h, b["weight"], b["bias"])
    z = scale * (y @ v["W"].T) @ points.T + bias
    return float((torch.logsumexp(z, 1) - z.gather(1, labels[:, None])[:, 0]).mean())


def test_example_gradients():
    # Each operator's results are off by at most (3 * 256 / 16 + 32) 2^-24 = 4.8e-6 of the magnitudes it adds up (the
    # longest sum's bound); 9 operators of the two blocks, forward and back, one behind the other: 18 * 4.8e-6 = 8.6e-5.
    # The differences' own error is below 1e-6 (h^2 of third derivatives, 1e-12 / h). All are held to 1e-4.
    from examples import query_tower
    t = query_tower.Tower(64, 24, 2, torch.Generator("cuda").manual_seed(3))
    g = torch.Generator().manual_seed(4)
    x, points = torch.randn(80, 64, generator=g), torch.randn(50, 24, generator=g)
    labels, bias = torch.randint(50, (80,), generator=g), torch.randn(50, generator=g)
    boa.softmax_xent(t(x.cuda()), points.cuda(), labels.cuda(), bias.cuda(), 0.5).backward()
    leaves = dict(norm0=t.norm[0], norm1=t.norm[1], W=t.W)
    for i, b in enumerate(t.blocks):
        leaves |= {f"{k}{i}": v for k, v in b.items()}
    values = {k: v.detach().double().cpu() for k, v in leaves.items()}
    rest = (x.double(), points.double(), labels, bias.double(), 0.5, 2)
    step = 1e-4
    for name, leaf in leaves.items():
        e = torch.randn(leaf.shape, generator=g, dtype=torch.float64)
        up, down = (plain_loss(values | {name: values[name] + s * e}, *rest) for s in (step, -step))
        terms = leaf.grad.double().cpu() * e
        assert abs(float(terms.sum()) - (up - down) / (2 * step)) <= 1e-4 * float(terms.abs().sum()), name


def test_example_runs_with_blocks():
    from examples import query_tower
    r = query_tower.main(["--steps", "12", "--points", "2000", "--blocks", "2"])
    assert math.isfinite(r["last"]) and torch.isfinite(r["served"]).all() and r["served"].shape == r["h"].shape
    assert all(torch.isfinite(m).all() and m.grad is None for m in r["tower"].hidden_matrices)
