"""Performance cases of the operators that fit a deeper query tower: matrix
products with bias, activation and residual in their epilogue (forward and
backward), the norms after and before a block with its gate and residual scale
(forward and backward), and the orthogonalisation of a weight's update.

A case is a dict of plain values. `run` computes each operator in elementary
torch operations in float32, rounded once at the end; with `own` set it calls
the package's operators instead. Widths follow the collections of
workloads/gen.py (32 to 768 dimensions, up to 1024) and hidden layers of 2 and 4 times
that, batches those of a tower: one query to tens of thousands of token states.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
STEPS = 5
COEFFICIENTS = (3.4445, -4.7750, 2.0315)

# the largest listed cost of each operator: a drawn case stays within it
MAX_LINEAR = 32_768 * 1024 * 4096
MAX_BLOCK = 65_536 * 1024
MAX_ORTH = 2048 * 2048 * 4096


def _linear(name, **kw):
    # M rows of K values times (N, K) weights; train: forward and backward, else forward only; gap: unused elements after each row
    return dict(dict(op="linear", name=name, dtype="bf16", act="gelu", bias=True, residual=False, train=True, gap=0), **kw)


def _block(name, **kw):
    # gate: "features" (one value a feature), "rows" (one a value), "none"; post: the block's output is normed too
    return dict(dict(op="block", name=name, dtype="bf16", params="bf16", norm="layer", gate="features", post=True, scale=1.0,
                     train=True), **kw)


def _orth(name, **kw):
    # count updates of rows x cols; rank: directions that carry most of the update
    return dict(dict(op="orth", name=name, dtype="bf16", count=1, rank=64), **kw)


def listed():
    return [
        # serving one query: the tower's hidden layer on a single state, latency
        _linear("linear-query", M=1, K=768, N=768, act="silu", train=False),
        # serving a few queries at once through the second layer of a block, with the residual stream
        _linear("linear-few", M=13, K=4096, N=1024, act="none", residual=True, train=False),
        # training on the token states of a batch of long texts: a block's first layer
        _linear("linear-tokens", M=32_768, K=1024, N=4096),
        # the block's second layer on a small batch, back to the residual stream
        _linear("linear-batch", M=1000, K=2048, N=768, act="none", residual=True),
        # a float32 tower on a training batch
        _linear("linear-batch-f32", M=10_000, K=768, N=1024, dtype="f32", act="silu"),
        # odd widths and rows inside a wider buffer
        _linear("linear-odd", M=9_973, K=413, N=777, dtype="f16", act="relu", residual=True, gap=3),
        # one query's state between two blocks: latency
        _block("block-query", rows=1, dim=768, train=False),
        # token states of a batch of long texts
        _block("block-tokens", rows=65_536, dim=1024, scale=0.81),
        # float32, odd widths, gates that another layer computed for each row
        _block("block-odd-f32", rows=9_973, dim=413, dtype="f32", params="f32", norm="rms", gate="rows"),
        # the small collection's projection, float32: latency
        _orth("orth-small", rows=32, cols=96, dtype="f32", rank=8),
        # float32 projections of four blocks
        _orth("orth-projections-f32", rows=768, cols=768, count=4, dtype="f32"),
        # a wide hidden layer
        _orth("orth-hidden", rows=4096, cols=2048),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "block", "orth"])
    if op == "linear":
        dtype = rng.choice(["bf16", "bf16", "f32", "f16"])
        K, N = (rng.choice([768, 1024, 2048, _log(rng, 32, 4096)]) for _ in range(2))
        most = min(65_536, (MAX_LINEAR if dtype != "f32" else MAX_LINEAR // 8) // (K * N), (1 << 28) // (K + N))
        c = _linear("", M=_log(rng, 1, most), K=K, N=N, dtype=dtype, act=rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"]),
                    bias=rng.random() < 0.7, residual=rng.random() < 0.5, train=rng.random() < 0.6, gap=rng.choice([0, 0, 8, 5]))
    elif op == "block":
        dtype = rng.choice(["bf16", "bf16", "f32", "f16"])
        dim = rng.choice([768, 1024, _log(rng, 32, 2048)])
        most = (MAX_BLOCK if dtype != "f32" else MAX_BLOCK // 2) // dim
        c = _block("", rows=_log(rng, 1, min(262_144, most)), dim=dim, dtype=dtype, params=rng.choice([dtype, "f32"]),
                   norm=rng.choice(["layer", "rms"]), gate=rng.choice(["features", "features", "rows", "none"]),
                   post=rng.random() < 0.6, scale=rng.choice([1.0, 0.81]), train=rng.random() < 0.7)
    else:
        dtype = rng.choice(["bf16", "f32"])
        rows, cols = (rng.choice([768, 1024, _log(rng, 16, 4096)]) for _ in range(2))
        lo = min(rows, cols)
        room = (MAX_ORTH if dtype != "f32" else MAX_ORTH // 4) // (lo * lo * max(rows, cols))
        if room < 1:
            rows, cols, lo, room = rows, 512, min(rows, 512), 1
        c = _orth("", rows=rows, cols=cols, count=rng.randint(1, max(1, min(8, room))), dtype=dtype,
                  rank=rng.randint(1, lo))
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs

def _gen(seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    return dev, lambda *s: torch.randn(*s, generator=g, device=dev)


def _inside(t, dt, gap):
    # t as rows of a buffer that has `gap` more elements a row
    wide = torch.zeros(t.shape[0], t.shape[1] + gap, device=t.device, dtype=dt)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def _states(normal, rows, d):
    # activations: per-feature offsets and spreads, a few features far larger than the others
    spread = torch.exp(0.5 * normal(d))
    spread[:: max(1, d // 4)] *= 8
    return normal(rows, d).mul_(spread).add_(0.3 * normal(d))


def prepare(case, seed):
    dev, normal = _gen(seed)
    op, dt = case["op"], DTYPES[case["dtype"]]
    s = dict(case)
    if op == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        # normed states, a few features larger; weights that keep their size
        x = normal(M, K)
        x[:, :: max(1, K // 4)] *= 4
        s.update(x=_inside(x, dt, case["gap"]), w=(normal(N, K) / math.sqrt(K)).to(dt),
                 b=(0.2 * normal(N)).to(dt) if case["bias"] else None,
                 r=_inside(normal(M, N), dt, case["gap"]) if case["residual"] else None)
        if case["train"]:
            s["dy"] = _inside(normal(M, N) * 1e-2, dt, case["gap"])
    elif op == "block":
        R, d, pt = case["rows"], case["dim"], DTYPES[case["params"]]
        s.update(x=_states(normal, R, d).to(dt), f=_states(normal, R, d).mul_(0.5).to(dt), eps=1e-5,
                 w=(1 + 0.2 * normal(d)).to(pt), b=(0.1 * normal(d)).to(pt), pw=None, pb=None, g=None)
        if case["post"]:
            s.update(pw=(1 + 0.2 * normal(d)).to(pt), pb=(0.1 * normal(d)).to(pt))
        if case["gate"] == "features":
            s["g"] = (0.3 * normal(d)).to(pt)
        elif case["gate"] == "rows":
            s["g"] = torch.sigmoid(normal(R, d)).to(dt)
        if case["train"]:
            s.update(dh=(normal(R, d) * 1e-2).to(dt), dy=(normal(R, d) * 1e-2).to(dt))
    else:
        C, R, L, k = case["count"], case["rows"], case["cols"], case["rank"]
        # the momentum of a layer's gradients: directions of falling weight over the batches' noise
        fall = (1 + torch.arange(k, device=dev)).float().rsqrt()
        s["u"] = (1e-3 * (torch.matmul(normal(C, R, k) * fall, normal(C, k, L)) / math.sqrt(k) + 0.1 * normal(C, R, L))).to(dt)
    return s


# ---------------------------------------------------------------------------
# one pass

def run(s):
    if own:
        return _run_own(s)
    return {"linear": _plain_linear, "block": _plain_block, "orth": _plain_orth}[s["op"]](s)


def _run_own(s):
    import paper_2609_16175_amd as boa
    if s["op"] == "linear":
        if not s["train"]:
            return boa.linear(s["x"], s["w"], s["b"], residual=s["r"], activation=s["act"])
        y, pre = boa.linear_forward(s["x"], s["w"], s["b"], residual=s["r"], activation=s["act"], keep=True)
        dx, dw, db = boa.linear_backward(s["dy"], s["x"], s["w"], pre, activation=s["act"], need=(True, True, s["bias"]))
        return dict(y=y, dx=dx, dw=dw, **(dict(db=db) if s["bias"] else {}))
    if s["op"] == "block":
        h, y, stats = boa.block_norm_forward(s["x"], s["f"], s["g"], scale=s["scale"], post=s["post"], post_weight=s["pw"],
                                             post_bias=s["pb"], weight=s["w"], bias=s["b"], norm=s["norm"], eps=s["eps"])
        if not s["train"]:
            return dict(h=h, y=y)
        r = boa.block_norm_backward(s["dh"], s["dy"], s["x"], s["f"], stats, s["g"], scale=s["scale"], post=s["post"],
                                    post_weight=s["pw"], post_bias=s["pb"], weight=s["w"], bias=s["b"], norm=s["norm"])
        out = dict(h=h, y=y, dx=r.dx, df=r.df, dw=r.dweight, db=r.dbias)
        if s["g"] is not None:
            out["dg"] = r.dgate
        if s["post"]:
            out.update(dpw=r.dpost_weight, dpb=r.dpost_bias)
        return out
    return boa.orthogonalize(s["u"], steps=STEPS, coefficients=COEFFICIENTS)


def _act(z, kind):
    if kind == "relu":
        return z * (z > 0)
    if kind == "silu":
        return z / (1 + torch.exp(-z))
    if kind == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if kind == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _slope(z, kind):
    if kind == "relu":
        return (z > 0).to(z.dtype)
    if kind == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    if kind == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z * z * z))
    return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)


def _plain_linear(s):
    x, w, dt = s["x"].float(), s["w"].float(), s["x"].dtype
    z = x @ w.t()
    if s["b"] is not None:
        z += s["b"].float()
    y = _act(z, s["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    y = y.to(dt)
    if not s["train"]:
        return y
    dz = s["dy"].float()
    if s["act"] != "none":
        dz = dz * _slope(z, s["act"])
    out = dict(y=y, dx=(dz @ w).to(dt), dw=(dz.t() @ x).to(dt))
    if s["b"] is not None:
        out["db"] = dz.sum(0).to(dt)
    return out


def _plain_norm(v, w, b, layer, eps):
    c = v - v.mean(1, keepdim=True) if layer else v
    r = torch.rsqrt((c * c).mean(1, keepdim=True) + eps)
    n = c * r
    return n, r, n * w.float() + b.float()


def _plain_norm_back(dy, n, r, w, layer):
    g = dy * w.float()
    d = g - n * (g * n).mean(1, keepdim=True)
    if layer:
        d -= g.mean(1, keepdim=True)
    return r * d, (dy * n).sum(0), dy.sum(0)


def _plain_block(s):
    dt, layer, gate = s["x"].dtype, s["norm"] == "layer", s["g"]
    x, f = s["x"].float(), s["f"].float()
    u = f
    if s["post"]:
        fn, fr, u = _plain_norm(f, s["pw"], s["pb"], layer, s["eps"])
    h = s["scale"] * x + (u if gate is None else gate.float() * u)
    hn, hr, y = _plain_norm(h, s["w"], s["b"], layer, s["eps"])
    out = dict(h=h.to(dt), y=y.to(dt))
    if not s["train"]:
        return out
    pt = s["w"].dtype
    dh, dw, db = _plain_norm_back(s["dy"].float(), hn, hr, s["w"], layer)
    dh += s["dh"].float()
    out.update(dx=(s["scale"] * dh).to(dt), dw=dw.to(pt), db=db.to(pt))
    du = dh
    if gate is not None:
        du = dh * gate.float()
        dg = dh * u
        out["dg"] = (dg if s["gate"] == "rows" else dg.sum(0)).to(gate.dtype)
    if s["post"]:
        du, dpw, dpb = _plain_norm_back(du, fn, fr, s["pw"], layer)
        out.update(dpw=dpw.to(pt), dpb=dpb.to(pt))
    out["df"] = du.to(dt)
    return out


def _plain_orth(s):
    x = s["u"].float()
    tall = x.shape[1] > x.shape[2]
    if tall:   # the smaller Gram matrix
        x = x.transpose(1, 2).contiguous()
    x = x / ((x * x).sum((1, 2), keepdim=True).sqrt() + 1e-7)
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        p = torch.matmul(x, x.transpose(1, 2))
        x = a * x + torch.matmul(b * p + c * torch.matmul(p, p), x)
    return (x.transpose(1, 2).contiguous() if tall else x).to(s["u"].dtype)


# ---------------------------------------------------------------------------
# the definitions in 64 bits

def _exact_linear(case, s):
    X, W, kind = s["x"].double(), s["w"].double(), case["act"]
    Z = torch.mm(X, W.T) if s["b"] is None else torch.addmm(s["b"].double(), X, W.T)
    cdf = torch.special.ndtr(Z) if kind == "gelu" else torch.sigmoid(Z) if kind == "silu" else None
    if kind == "gelu_tanh":   # (1 + tanh q) / 2 = sigmoid(2 q)
        q2 = 2 * math.sqrt(2 / math.pi) * Z * (1 + 0.044715 * Z.square())
        cdf = torch.sigmoid(q2)
    Y = Z if kind == "none" else Z.clamp(min=0) if kind == "relu" else Z * cdf
    if s["r"] is not None:
        Y = Y + s["r"].double()
    if not case["train"]:
        return Y
    D = s["dy"].double()
    if kind == "relu":
        D = torch.where(Z > 0, D, torch.zeros_like(D))
    elif kind == "silu":
        D = D * (cdf + Z * cdf * (1 - cdf))
    elif kind == "gelu":
        D = D * (cdf + Z * torch.exp(-Z.square() / 2) / math.sqrt(2 * math.pi))
    elif kind == "gelu_tanh":
        D = D * (cdf + Z * cdf * (1 - cdf) * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * Z.square()))
    out = dict(y=Y, dx=torch.mm(D, W), dw=torch.mm(D.T, X))
    if s["b"] is not None:
        out["db"] = D.sum(0)
    return out


def _exact_unit(V, layer, eps):
    # unit rows and the deviation they were divided by
    if layer:
        var, mu = torch.var_mean(V, dim=1, unbiased=False, keepdim=True)
        sd = (var + eps).sqrt()
        return (V - mu) / sd, sd
    sd = (V.square().mean(1, keepdim=True) + eps).sqrt()
    return V / sd, sd


def _exact_unit_back(DY, Z, sd, W, layer):
    U, d = DY * W, DY.shape[1]
    T = d * U - Z * (U * Z).sum(1, keepdim=True)
    if layer:
        T = T - U.sum(1, keepdim=True)
    return T / (d * sd)


def _exact_block(case, s):
    layer, eps, k = case["norm"] == "layer", s["eps"], case["scale"]
    D = {n: None if s.get(n) is None else s[n].double() for n in ("x", "f", "g", "w", "b", "pw", "pb", "dh", "dy")}
    U = D["f"]
    if case["post"]:
        FZ, fsd = _exact_unit(U, layer, eps)
        U = torch.addcmul(D["pb"], FZ, D["pw"])
    G = torch.ones_like(U[0]) if D["g"] is None else D["g"]
    H = torch.addcmul(D["x"] * k, G.expand_as(U), U)
    HZ, hsd = _exact_unit(H, layer, eps)
    out = dict(h=H, y=torch.addcmul(D["b"], HZ, D["w"]))
    if case["train"]:
        DH = D["dh"] + _exact_unit_back(D["dy"], HZ, hsd, D["w"], layer)
        out.update(dx=k * DH, dw=torch.einsum("rd,rd->d", D["dy"], HZ), db=D["dy"].sum(0))
        if case["gate"] == "rows":
            out["dg"] = DH * U
        elif case["gate"] == "features":
            out["dg"] = torch.einsum("rd,rd->d", DH, U)
        DU = DH * G
        if case["post"]:
            out.update(dpw=torch.einsum("rd,rd->d", DU, FZ), dpb=DU.sum(0))
            DU = _exact_unit_back(DU, FZ, fsd, D["pw"], layer)
        out["df"] = DU
    return out


def _exact_orth(case, s):
    # X (a + b S + c S^2) with S = X^T X the smaller of the two Gram matrices, one update after the other
    a, b, c = COEFFICIENTS
    out = []
    for U in s["u"].double():
        X = U if case["rows"] >= case["cols"] else U.T
        X = X / (torch.linalg.matrix_norm(X) + 1e-7)
        eye = torch.eye(X.shape[1], dtype=torch.float64, device=X.device)
        for _ in range(STEPS):
            S = torch.mm(X.T, X)
            X = torch.mm(X, a * eye + torch.mm(S, b * eye + c * S))
        out.append(X if case["rows"] >= case["cols"] else X.T)
    return torch.stack(out)


def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "block": _exact_block, "orth": _exact_orth}[case["op"]](case, s)


# ---------------------------------------------------------------------------

def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        out = M * N * (2 if case["residual"] else 1)
        bias = N if case["bias"] else 0
        n = M * K + N * K + bias + out
        if case["train"]:
            n += M * N + M * K + N * K + bias
        return dict(bytes=n * e, flops=2.0 * M * K * N * (3 if case["train"] else 1))
    if case["op"] == "block":
        n, d, pe = case["rows"] * case["dim"], case["dim"], BYTES[case["params"]]
        vectors = 2 + (2 if case["post"] else 0) + (1 if case["gate"] == "features" else 0)
        full = 1 if case["gate"] == "rows" else 0
        b = (4 + full) * n * e + vectors * d * pe
        if case["train"]:
            b += (4 + full) * n * e + vectors * d * pe
        return dict(bytes=b, flops=(50 if case["train"] else 16) * n)
    C, m, n = case["count"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    # the two Gram matrices are symmetric: half of each product
    return dict(bytes=2 * C * m * n * e, flops=1.0 * C * STEPS * (m * m * n + m * m * m + 2 * m * m * n))
