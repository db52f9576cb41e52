"""Fit a query tower to an index and serve it.

An encoder's states x (here: points of the collection, mixed into a wider
space with noise) become query vectors h = W layer_norm(x). The tower is fitted
so that the index finds a state's own point: softmax cross entropy over all
points as classes, with the negative squared distance of the search as logit
(scale = 2 t, bias = -t |p|^2; t |h|^2 is the same for every class). Serving
takes one state at a time: layer norm, then W in 4 bits, then the search.

With --blocks the tower has residual blocks between the two: h <- h + gate V
gelu(U y), y <- layer_norm(h). Their matrices learn from orthogonalised
momenta, everything else from Adam.

    python examples/query_tower.py [--steps 200] [--blocks 2]
"""
import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import numpy as np  # noqa: E402
import torch  # noqa: E402

import paper_2609_16175_amd as boa  # noqa: E402
from workloads import gen, rows4  # noqa: E402


def found(index, queries, labels, wl):
    """Share of the queries whose own point is among the k results."""
    ranges = torch.tensor([-2 ** 31, 2 ** 31 - 1], dtype=torch.int32, device="cuda").expand(len(queries), wl.m, 2)
    ids = index.search(queries.float(), ranges, wl.k, L0=32, Lmax=wl.Lmax, eps=0.0).ids
    return float((ids == labels[:, None]).any(1).float().mean())


class Tower:
    """W of the last layer norm of a residual stream, which `blocks` blocks of `states` x 4 `states` weights add to."""

    def __init__(self, states, d, blocks, g):
        def leaf(t):
            return t.requires_grad_()

        def matrix(rows, cols):
            return leaf(torch.randn(rows, cols, generator=g, device="cuda") / cols ** 0.5)

        def vector(n, value):
            return leaf(torch.full((n,), value, device="cuda"))

        self.norm = vector(states, 1.0), vector(states, 0.0)
        self.W = matrix(d, states)
        self.blocks = [dict(up=matrix(4 * states, states), up_bias=vector(4 * states, 0.0), down=matrix(states, 4 * states),
                            down_bias=vector(states, 0.0), gate=vector(states, 0.2), weight=vector(states, 1.0),
                            bias=vector(states, 0.0)) for _ in range(blocks)]
        self.hidden_matrices = [b[k] for b in self.blocks for k in ("up", "down")]
        self.momenta = [torch.zeros_like(m) for m in self.hidden_matrices]
        self.others = [*self.norm, self.W, *(v for b in self.blocks for k, v in b.items() if k not in ("up", "down"))]

    def hidden(self, x):
        """What W is applied to."""
        h, y = x, boa.layer_norm(x, *self.norm)
        for b in self.blocks:
            f = boa.linear(boa.linear(y, b["up"], b["up_bias"], activation="gelu"), b["down"], b["down_bias"])
            h, y = boa.block_norm(h, f, b["gate"], weight=b["weight"], bias=b["bias"])
        return y

    def __call__(self, x):
        return boa.linear(self.hidden(x), self.W)

    @torch.no_grad()
    def step_hidden(self, lr=0.02, beta=0.9):
        """Each hidden matrix a step against its orthogonalised momentum."""
        for m, v in zip(self.hidden_matrices, self.momenta):
            v.mul_(beta).add_(m.grad)
            m.sub_(boa.orthogonalize(v), alpha=lr * max(1.0, m.shape[0] / m.shape[1]) ** 0.5)
            m.grad = None


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--points", type=int, default=10_000)
    ap.add_argument("--states", type=int, default=96, help="width of the encoder's states")
    ap.add_argument("--blocks", type=int, default=0, help="residual blocks of the tower")
    a = ap.parse_args(argv)
    wl = gen.TINY.scaled(a.points, nq=64)
    data = gen.generate(wl)
    types = np.array(wl.attr_dtypes, dtype=np.int32)
    index = boa.Index(data.vectors, data.attrs, types, None, -1, R=wl.R)

    g = torch.Generator("cuda").manual_seed(7)
    points = torch.from_numpy(data.vectors).cuda()
    n, d = points.shape
    mix = torch.randn(d, a.states, generator=g, device="cuda") / d ** 0.5
    shift = torch.randn(a.states, generator=g, device="cuda")

    def states(labels):   # what an encoder gives for a text about each point
        return points[labels] @ mix + shift + 0.1 * torch.randn(len(labels), a.states, generator=g, device="cuda")

    tower = Tower(a.states, d, a.blocks, g)
    opt = torch.optim.Adam(tower.others, lr=2e-2)
    t = 2.0
    bias = -t * points.square().sum(1)

    held = torch.randint(n, (256,), generator=g, device="cuda")
    held_x = states(held)

    with torch.no_grad():
        first = float(boa.softmax_xent(tower(held_x), points, held, bias, 2 * t))
        print(f"before: loss {first:.3f}, own point found {found(index, tower(held_x), held, wl):.3f}", flush=True)
    for step in range(a.steps):
        labels = torch.randint(n, (512,), generator=g, device="cuda")
        loss = boa.softmax_xent(tower(states(labels)), points, labels, bias, 2 * t)
        opt.zero_grad()
        loss.backward()
        opt.step()
        tower.step_hidden()
        if (step + 1) % 50 == 0:
            print(f"step {step + 1}: loss {float(loss.detach()):.3f}", flush=True)
    with torch.no_grad():
        h = tower(held_x)
        last = float(boa.softmax_xent(h, points, held, bias, 2 * t))
        whole = found(index, h, held, wl)
        # serving: one state at a time through 4-bit weights
        codes, scales, offsets = rows4.quantize(tower.W, group=32)
        one = [boa.matvec_4bit(tower.hidden(x[None]), codes, scales, offsets) for x in held_x]
        served = torch.cat(one)
        in4 = found(index, served, held, wl)
    print(f"after: loss {last:.3f}, own point found {whole:.3f}, with 4-bit weights {in4:.3f}", flush=True)
    index.close()
    return dict(first=first, last=last, found=whole, found_4bit=in4, h=h, served=served, W=tower.W.detach(), norm=tower.norm,
                x=held_x, tower=tower)


if __name__ == "__main__":
    main()
