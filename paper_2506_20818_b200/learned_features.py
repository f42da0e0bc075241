"""Link prediction on a graph without node features: a learned embedding table and a two-layer transform, trained with
orthogonalised updates.

    python -m paper_2506_20818_b200.learned_features --nodes 20000 --steps 200

Every node has a row of a table E.  A step draws a batch of edges and one negative each, looks the rows of its three
endpoints up (lp_embed), runs them through H = ReLU(x W1 + b1), Z = H W2 + b2 (lp_op_linear), scores pairs by the dot
product, takes the binary cross-entropy, and goes back through the same operators: lp_op_weight_grad for W1 and W2,
lp_embed_grad for E.  E, W1, b1, W2, b2 lie in one flat vector and one call of lp_muon_step updates it: W1 and W2 with
orthogonalised momentum, the table and the biases with Adam.
"""
from __future__ import annotations

import argparse
import json
import math


class LearnedFeatures:
    """Table, transform and optimiser state on one GPU; `ctx` needs a loaded graph (for the negatives)."""

    def __init__(self, ctx, nodes: int, width: int = 64, hidden: int = 128, out: int = 64, seed: int = 0):
        import torch

        self.ctx, self.torch = ctx, torch
        self.nodes, self.width, self.hidden, self.out = nodes, width, hidden, out
        dev = f"cuda:{ctx.device}"
        gen = torch.Generator(device=dev).manual_seed(seed)
        sizes = [("E", nodes, width), ("W1", width, hidden), ("b1", 1, hidden), ("W2", hidden, out), ("b2", 1, out)]
        self.offset, at = {}, 0
        for name, rows, cols in sizes:
            self.offset[name] = (at, rows, cols)
            at += rows * cols
        self.params = torch.zeros(at, device=dev)
        self.part(self.params, "E").normal_(generator=gen).mul_(1.0 / math.sqrt(width))
        for name in ("W1", "W2"):
            w = self.part(self.params, name)
            w.normal_(generator=gen).mul_(math.sqrt(2.0 / sum(w.shape)))
        self.grads, self.momentum, self.second = (torch.zeros_like(self.params) for _ in range(3))
        self.matrices = [self.offset["W1"], self.offset["W2"]]
        self.scale = math.sqrt(width)
        self.t = 0

    def part(self, flat, name):
        at, rows, cols = self.offset[name]
        return flat[at:at + rows * cols].view(rows, cols)

    def forward(self, ids):
        """Rows of the table and the activations of every id."""
        t = self.torch
        p = {n: self.part(self.params, n) for n in self.offset}
        w1, w2 = p["W1"].to(t.bfloat16), p["W2"].to(t.bfloat16)
        x = self.ctx.embed(p["E"], ids, scale=self.scale, out_dtype=t.bfloat16)
        h = self.ctx.op_linear(x, w1, p["b1"].reshape(-1).contiguous(), relu=True)
        z = self.ctx.op_linear(h, w2, p["b2"].reshape(-1).contiguous())
        return x, h, z, w1, w2

    def step(self, src, dst, neg, lr: float = 0.02, adam_lr: float = 3e-3) -> float:
        """One update on the edges (src, dst) and the non-edges (src, neg); returns the loss before it."""
        t = self.torch
        B = src.numel()
        ids = t.cat((src, dst, neg))
        x, h, z, w1, w2 = self.forward(ids)
        zs, zd, zn = (part.float() for part in z.view(3, B, self.out))
        pos, negs = (zs * zd).sum(1), (zs * zn).sum(1)
        loss = (t.nn.functional.softplus(-pos).sum() + t.nn.functional.softplus(negs).sum()) / (2 * B)
        gp, gn = ((t.sigmoid(pos) - 1.0) / (2 * B))[:, None], (t.sigmoid(negs) / (2 * B))[:, None]
        dz = t.cat((gp * zd + gn * zn, gp * zs, gn * zs))
        g = {n: self.part(self.grads, n) for n in self.offset}
        dz16 = dz.to(t.bfloat16)
        g["b2"].copy_(dz.sum(0, keepdim=True))
        g["W2"].copy_(self.ctx.op_weight_grad(h, dz16))
        dh = self.ctx.op_linear(dz16, w2, trans_b=True) * (h > 0)
        g["b1"].copy_(dh.float().sum(0, keepdim=True))
        g["W1"].copy_(self.ctx.op_weight_grad(x, dh))
        dx = self.ctx.op_linear(dh, w1, trans_b=True)
        self.ctx.embed_grad(dx, ids, self.nodes, scale=self.scale, grad=g["E"])
        self.t += 1
        self.ctx.muon_step(self.params, self.momentum, self.second, self.grads, t=self.t, matrices=self.matrices, lr=lr, adam_lr=adam_lr)
        return float(loss)


def main() -> None:
    ap = argparse.ArgumentParser()
    ap.add_argument("--nodes", type=int, default=20_000)
    ap.add_argument("--mean-degree", type=float, default=12.0)
    ap.add_argument("--width", type=int, default=64)
    ap.add_argument("--batch", type=int, default=8192)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--lr", type=float, default=0.02)
    ap.add_argument("--seed", type=int, default=0)
    args = ap.parse_args()

    import torch
    import workloads as wl
    from . import Context

    g = wl.chung_lu(args.nodes, args.mean_degree, 2.1, seed=args.seed)
    ctx = Context(0)
    ctx.load_graph(g.n, g.rowptr, g.col, None, wl.node_features(g.n, 8, args.seed))
    u, v = (torch.from_numpy(x).to("cuda:0") for x in wl.undirected_edge_list(g))
    model = LearnedFeatures(ctx, g.n, args.width, seed=args.seed)
    gen = torch.Generator(device="cuda:0").manual_seed(args.seed)
    losses = []
    for step in range(args.steps):
        pick = torch.randint(0, u.numel(), (min(args.batch, u.numel()),), device="cuda:0", generator=gen)
        src, dst = u[pick].contiguous(), v[pick].contiguous()
        _, neg = ctx.sample_negatives(args.seed, step, 1, src)
        losses.append(model.step(src, dst, neg, lr=args.lr))
    ctx.stats()
    tail = losses[-max(1, len(losses) // 10):]
    print(json.dumps({"nodes": g.n, "edges": int(u.numel()), "width": args.width, "steps": args.steps, "first_loss": losses[0], "last_loss": sum(tail) / len(tail)}))
    ctx.close()


if __name__ == "__main__":
    main()
