"""Performance cases of the query-tower operators: layer norm (forward and
backward), softmax cross entropy over the points of an index (loss and
gradients), and matrix-vector products with 4-bit rows.

A case is a dict of plain values. `run` computes each operator in elementary
torch operations in float32, rounded once at the end; with `own` set it calls
the package's operators instead. Sizes follow the collections of
workloads/gen.py (10,000 to 1,000,000 points, 32 to 768 dimensions, batches
of 1 to 10,000 queries).
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}

# the largest listed cost of each operator: a drawn case stays within it
MAX_NORM = 65_536 * 1024
MAX_LOGITS = 2048 * 1_000_000
MAX_XENT = MAX_LOGITS * 128
MAX_ROWS4 = 1_000_000 * 768


def _norm(name, **kw):
    # rows x dim activations; train: forward and backward, else forward only; gap: unused elements after each row
    return dict(dict(op="norm", name=name, dtype="bf16", train=True, gap=0), **kw)


def _xent(name, **kw):
    # batch rows against `classes` points; grads: "none" (losses of an evaluation), "h" (the points stay as they are), "all"
    return dict(dict(op="xent", name=name, dtype="bf16", grads="all", bias=True, scale=20.0, ignored=0.02), **kw)


def _rows4(name, **kw):
    # batch vectors of K values against `rows` rows of 4-bit codes
    return dict(dict(op="rows4", name=name, dtype="bf16", scales="bf16", group=32, offsets=True), **kw)


def listed():
    return [
        # one query's hidden state before the projection: latency
        _norm("norm-query", rows=1, dim=768, train=False),
        # a training batch of the dblp-like width in float32
        _norm("norm-batch-f32", rows=10_000, dim=768, dtype="f32"),
        # token states of a batch of long texts, the widest rows an index takes
        _norm("norm-tokens", rows=65_536, dim=1024),
        # odd widths and rows inside a wider buffer
        _norm("norm-odd", rows=9_973, dim=413, dtype="f16", gap=3),
        # fitting a query tower to the small collection, float32 throughout
        _xent("xent-tiny", batch=100, classes=10_000, dim=32, dtype="f32"),
        # the loss of one held-out query over a million descriptors
        _xent("xent-eval-one", batch=1, classes=1_000_000, dim=128, grads="none"),
        # a query tower against a fixed index of image features, a number of points no tile divides
        _xent("xent-queries", batch=1_000, classes=999_983, dim=96, grads="h"),
        # the largest: points trained with the tower, a million of them
        _xent("xent-points", batch=2_048, classes=1_000_000, dim=128),
        # text embeddings, float32, points and tower trained
        _xent("xent-text-f32", batch=777, classes=100_003, dim=768, dtype="f32", bias=False),
        # the tower's projection for one query: latency
        _rows4("rows4-projection", batch=1, rows=768, K=768),
        # one query against every text embedding in 4 bits
        _rows4("rows4-scan", batch=1, rows=1_000_000, K=768, group=64, offsets=False),
        # a few float32 queries at once against the descriptors, odd number of rows
        _rows4("rows4-few-f32", batch=5, rows=999_983, K=128, dtype="f32", scales="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "xent", "xent", "rows4"])
    if op == "norm":
        dim = _log(rng, 32, 1024)
        c = _norm("", rows=_log(rng, 1, min(262_144, MAX_NORM // dim)), dim=dim, dtype=rng.choice(["f32", "bf16", "f16"]),
                  train=rng.random() < 0.7, gap=rng.choice([0, 0, 8, 5]))
        if c["dtype"] == "f32":
            c["rows"] = max(1, min(c["rows"], MAX_NORM // 2 // dim))
    elif op == "xent":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        dim = rng.choice([32, 96, 128, 768, _log(rng, 16, 1024)])
        classes = _log(rng, 1_000, 1_000_000)
        top = min(MAX_LOGITS // classes, MAX_XENT // (classes * dim))
        batch = _log(rng, 1, max(1, min(10_000, top if dtype == "bf16" else top // 4)))
        c = _xent("", batch=batch, classes=classes, dim=dim, dtype=dtype, grads=rng.choice(["none", "h", "all", "all"]),
                  bias=rng.random() < 0.5, scale=rng.choice([1.0, 10.0, 20.0]), ignored=rng.choice([0.0, 0.02, 0.3]))
    else:
        group = rng.choice([32, 64, 128])
        K = group * rng.randint(1, 1024 // group)
        c = _rows4("", batch=rng.randint(1, 16), rows=_log(rng, 300, MAX_ROWS4 // K if K > 768 else 1_000_000), K=K,
                   group=group, dtype=rng.choice(["bf16", "f32", "f16"]), scales=rng.choice(["bf16", "f32"]),
                   offsets=rng.random() < 0.5)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs

def _gen(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    return dev, g, lambda *s: torch.randn(*s, generator=g, device=dev)


def prepare(case, seed):
    dev, g, normal = _gen(case, seed)
    op = case["op"]
    dt = DTYPES[case["dtype"]]
    s = dict(case)
    if op == "norm":
        R, d = case["rows"], case["dim"]
        # activations: per-feature offsets and spreads, a few features far larger than the others
        spread = torch.exp(0.5 * normal(d))
        spread[:: max(1, d // 4)] *= 8
        wide = torch.empty(R, d + case["gap"], device=dev, dtype=dt)
        wide.copy_(normal(R, d + case["gap"]))
        x = wide[:, :d]
        x.copy_(x.float() * spread + 0.3 * normal(d))
        s.update(x=x, w=(1 + 0.2 * normal(d)).to(dt), b=(0.1 * normal(d)).to(dt), eps=1e-5)
        if case["train"]:
            s["dy"] = (normal(R, d) * 1e-2).to(dt)
    elif op == "xent":
        B, V, d = case["batch"], case["classes"], case["dim"]
        # unit rows around clusters; a query is its point with noise
        centres = normal(max(4, V // 1000), d)
        pts = normal(V, d)
        pts.mul_(0.7).add_(centres[torch.randint(centres.shape[0], (V,), generator=g, device=dev)])
        pts.div_(pts.norm(dim=1, keepdim=True))
        labels = torch.randint(V, (B,), generator=g, device=dev)
        h = pts[labels] + 0.5 * normal(B, d) / math.sqrt(d)
        h.div_(h.norm(dim=1, keepdim=True))
        bias = None
        if case["bias"]:
            # small popularity offsets, and some points left out that no query asks for
            bias = 0.3 * normal(V)
            out = torch.rand(V, generator=g, device=dev) < 0.001
            out[labels] = False
            bias[out] = -math.inf
        drop = torch.rand(B, generator=g, device=dev) < case["ignored"]
        if B > 1:
            drop[0] = False
            labels = torch.where(drop, torch.full_like(labels, -1), labels)
        s.update(h=h.to(dt), pts=pts.to(dt), labels=labels, class_bias=bias)
    else:
        M, N, K, G = case["batch"], case["rows"], case["K"], case["K"] // case["group"]
        sdt = DTYPES[case["scales"]]
        # bell-shaped codes, as rounding normal weights gives them
        codes = torch.empty(N, K // 2, device=dev, dtype=torch.uint8)
        step = max(1, (1 << 27) // K)
        for i in range(0, N, step):
            q = (normal(min(step, N - i), K) * 2.6 + 7.6).round_().clamp_(0, 15).to(torch.uint8)
            codes[i:i + step] = q[:, 0::2] | (q[:, 1::2] << 4)
        scale = (0.01 * torch.exp(0.3 * normal(N, G))).to(sdt)
        s.update(x=normal(M, K).to(dt), codes=codes, s=scale,
                 o=(-8 * scale.float() * (1 + 0.05 * normal(N, G))).to(sdt) if case["offsets"] else None)
    return s


# ---------------------------------------------------------------------------
# one pass

def run(s):
    if own:
        return _run_own(s)
    return {"norm": _plain_norm, "xent": _plain_xent, "rows4": _plain_rows4}[s["op"]](s)


def _run_own(s):
    import paper_2609_16175_amd as boa
    if s["op"] == "norm":
        y, mean, rstd = boa.layer_norm_forward(s["x"], s["w"], s["b"], s["eps"])
        if not s["train"]:
            return y
        dx, dw, db = boa.layer_norm_backward(s["dy"], s["x"], s["w"], mean, rstd)
        return dict(y=y, dx=dx, dw=dw, db=db)
    if s["op"] == "xent":
        if s["grads"] == "none":
            return boa.softmax_xent(s["h"], s["pts"], s["labels"], bias=s["class_bias"], scale=s["scale"], reduction="none")
        r = boa.softmax_xent_grad(s["h"], s["pts"], s["labels"], bias=s["class_bias"], scale=s["scale"],
                                  rows_grad=s["grads"] == "all", bias_grad=s["grads"] == "all" and s["bias"])
        out = dict(loss=r.loss, dh=r.dh)
        if s["grads"] == "all":
            out["drows"] = r.drows
            if s["bias"]:
                out["dbias"] = r.dbias
        return out
    return boa.matvec_4bit(s["x"], s["codes"], s["s"], s["o"], group=s["group"])


def _plain_norm(s):
    x, w = s["x"].float(), s["w"].float()
    dt = s["x"].dtype
    c = x - x.mean(1, keepdim=True)
    r = torch.rsqrt((c * c).mean(1, keepdim=True) + s["eps"])
    xh = c * r
    y = (xh * w + s["b"].float()).to(dt)
    if not s["train"]:
        return y
    dy = s["dy"].float()
    g = dy * w
    dx = r * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dict(y=y, dx=dx.to(dt), dw=(dy * xh).sum(0).to(dt), db=dy.sum(0).to(dt))


def _plain_xent(s):
    h, c, labels = s["h"].float(), s["pts"].float(), s["labels"]
    dt = s["h"].dtype
    l = s["scale"] * (h @ c.t())
    if s["class_bias"] is not None:
        l += s["class_bias"]
    valid = labels >= 0
    at = labels.clamp(min=0)[:, None]
    m = l.amax(1, keepdim=True)
    picked = l.gather(1, at)
    p = torch.exp(l.sub_(m))
    z = p.sum(1, keepdim=True)
    loss = torch.where(valid, (m + torch.log(z) - picked)[:, 0], torch.zeros_like(z[:, 0]))
    if s["grads"] == "none":
        return loss
    n = valid.sum().clamp(min=1).float()
    p.div_(z)
    p.scatter_add_(1, at, torch.full_like(z, -1.0))
    p.mul_((valid.float() / n)[:, None])
    out = dict(loss=loss.sum() / n, dh=(s["scale"] * (p @ c)).to(dt))
    if s["grads"] == "all":
        out["drows"] = (s["scale"] * (p.t() @ h)).to(dt)
        if s["class_bias"] is not None:
            out["dbias"] = p.sum(0)
    return out


def _plain_rows4(s):
    codes, G = s["codes"], s["s"].shape[1]
    N, K = codes.shape[0], codes.shape[1] * 2
    q = torch.stack((codes & 15, codes >> 4), dim=2).reshape(N, G, K // G).float()
    sc = s["s"].float()[:, :, None]
    w = sc * (q - 8) if s["o"] is None else sc * q + s["o"].float()[:, :, None]
    return (s["x"].float() @ w.reshape(N, K).t()).to(s["x"].dtype)


# ---------------------------------------------------------------------------
# the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        X, W, Bs = s["x"].double(), s["w"].double(), s["b"].double()
        var, mu = torch.var_mean(X, dim=1, unbiased=False, keepdim=True)
        sd = (var + s["eps"]).sqrt()
        Z = (X - mu) / sd
        y = torch.addcmul(Bs, Z, W)
        if not case["train"]:
            return y
        DY = s["dy"].double()
        U = DY * W
        d = X.shape[1]
        dx = (d * U - U.sum(1, keepdim=True) - Z * (U * Z).sum(1, keepdim=True)) / (d * sd)
        return dict(y=y, dx=dx, dw=torch.einsum("rd,rd->d", DY, Z), db=DY.sum(0))
    if case["op"] == "xent":
        H, C, sc, lab = s["h"].double(), s["pts"].double(), case["scale"], s["labels"]
        off = s["class_bias"].double() if s["class_bias"] is not None else None
        B, V = case["batch"], case["classes"]
        keep = [i for i, v in enumerate(lab.tolist()) if v >= 0]
        losses = torch.zeros(B, dtype=torch.float64, device=H.device)
        full = case["grads"] != "none"
        dh, dc = torch.zeros_like(H), torch.zeros_like(C) if case["grads"] == "all" else None
        dbias = torch.zeros(V, dtype=torch.float64, device=H.device)
        step = max(1, int(2.5e8) // V)
        for i in range(0, len(keep), step):
            at = torch.tensor(keep[i:i + step], device=H.device)
            z = torch.mm(H[at], C.T) * sc
            if off is not None:
                z = z + off
            logp = torch.log_softmax(z, dim=1)
            rows = torch.arange(len(at), device=H.device)
            losses[at] = -logp[rows, lab[at]]
            if not full:
                continue
            q = logp.exp_()
            q[rows, lab[at]] -= 1.0
            q /= len(keep)
            dh[at] = torch.mm(q, C) * sc
            if dc is not None:
                dc.addmm_(q.T, H[at], alpha=sc)
                dbias += q.sum(0)
        if not full:
            return losses
        out = dict(loss=losses.sum() / max(1, len(keep)), dh=dh)
        if dc is not None:
            out["drows"] = dc
            if off is not None:
                out["dbias"] = dbias
        return out
    X, N, K, g = s["x"].double(), case["rows"], case["K"], case["group"]
    out = torch.zeros(X.shape[0], N, dtype=torch.float64, device=X.device)
    for j in range(K // g):
        part = s["codes"][:, j * g // 2:(j + 1) * g // 2]
        even, odd = (part % 16).double(), (part // 16).double()
        xs = X[:, j * g:(j + 1) * g]
        dot = torch.mm(xs[:, 0::2], even.T) + torch.mm(xs[:, 1::2], odd.T)
        scale = s["s"][:, j].double()
        shift = -8 * scale if s["o"] is None else s["o"][:, j].double()
        out += dot * scale + xs.sum(1, keepdim=True) * shift
    return out


# ---------------------------------------------------------------------------

def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "norm":
        n, d = case["rows"] * case["dim"], case["dim"]
        return dict(bytes=(4 * n + 4 * d) * e if case["train"] else (2 * n + 2 * d) * e, flops=(20 if case["train"] else 8) * n)
    if case["op"] == "xent":
        B, V, d = case["batch"], case["classes"], case["dim"]
        grads = {"none": 0, "h": 1, "all": 2}[case["grads"]]
        bytes_ = (B + V) * d * e + 8 * B + (4 * V if case["bias"] else 0)
        bytes_ += 4 * B if not grads else 4 + B * d * e + (V * d * e + (4 * V if case["bias"] else 0) if grads == 2 else 0)
        return dict(bytes=bytes_, flops=2.0 * (1 + grads) * B * V * d)
    M, N, K, G = case["batch"], case["rows"], case["K"], case["K"] // case["group"]
    per = BYTES[case["scales"]] * (2 if case["offsets"] else 1)
    return dict(bytes=N * K // 2 + N * G * per + (M * K + M * N) * e, flops=2.0 * M * N * K)
