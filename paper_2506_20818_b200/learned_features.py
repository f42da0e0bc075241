"""Link prediction on a graph without node features: a learned embedding table and a two-layer transform, trained with
orthogonalised updates.

    python -m paper_2506_20818_b200.learned_features --nodes 20000 --steps 200

Every node has a row of a table E.  A step draws a batch of edges and one negative each, looks the rows of its three
endpoints up (lp_embed), runs them through H = ReLU(x W1 + b1), Z = H W2 + b2 (lp_op_linear), scores pairs by the dot
product, takes the binary cross-entropy, and goes back through the same operators: lp_op_weight_grad for W1 and W2,
lp_embed_grad for E.  E, W1, b1, W2, b2 lie in one flat vector and one call of lp_muon_step updates it: W1 and W2 with
orthogonalised momentum, the table and the biases with Adam.

    python -m paper_2506_20818_b200.learned_features --types 4 --blocks 2 --dropout 0.1

puts residual blocks in the place of the first transform, each with one weight matrix per node type (types are runs of node ids,
as a partition or a typed graph numbers them):
    n = norm(s),  s <- s + gate * dropout(norm(ReLU(n W[type] + b[type])))
A batch is sorted by id, so that its rows are sorted by type; lp_grouped_linear and lp_grouped_weight_grad multiply,
lp_residual_norm ends a block and begins the next in one pass, and lp_residual_norm_grad draws the dropout again instead of
keeping a mask.
"""
from __future__ import annotations

import argparse
import json
import math


class LearnedFeatures:
    """Table, transform and optimiser state on one GPU; `ctx` needs a loaded graph (for the negatives)."""

    def __init__(self, ctx, nodes: int, width: int = 64, hidden: int = 128, out: int = 64, seed: int = 0, types: int = 1, blocks: int = 0, dropout: float = 0.0):
        import torch

        if types < 1 or blocks < 0 or not 0.0 <= dropout <= 1.0:
            raise ValueError("LearnedFeatures: at least one type, no negative number of blocks, dropout in [0, 1]")
        if blocks == 0 and (types != 1 or dropout != 0.0):
            raise ValueError("LearnedFeatures: types and dropout belong to the residual blocks, and there are none")
        self.ctx, self.torch = ctx, torch
        self.nodes, self.width, self.hidden, self.out = nodes, width, hidden, out
        self.types, self.blocks, self.dropout, self.seed = types, blocks, dropout, seed
        dev = f"cuda:{ctx.device}"
        gen = torch.Generator(device=dev).manual_seed(seed)
        if blocks > 0:
            # W, b: the matrices and biases of the types, norms: before each block and the last transform, after each block
            sizes = [("E", nodes, width), ("W2", width, out), ("b2", 1, out), ("pre", blocks + 1, width), ("post", blocks, width), ("gate", blocks, width)]
            sizes += [(f"{n}{i}", types * rows, width) for i in range(blocks) for n, rows in (("W", width), ("b", 1))]
        else:
            sizes = [("E", nodes, width), ("W1", width, hidden), ("b1", 1, hidden), ("W2", hidden, out), ("b2", 1, out)]
        self.offset, at = {}, 0
        for name, rows, cols in sizes:
            self.offset[name] = (at, rows, cols)
            at += rows * cols
        self.params = torch.zeros(at, device=dev)
        self.part(self.params, "E").normal_(generator=gen).mul_(1.0 / math.sqrt(width))
        for name in (n for n, _, _ in sizes if n[0] == "W"):
            w = self.part(self.params, name)
            w.normal_(generator=gen).mul_(math.sqrt(2.0 / (w.shape[0] // (types if blocks > 0 and name != "W2" else 1) + w.shape[1])))
        for name in ("pre", "post", "gate") if blocks > 0 else ():
            self.part(self.params, name).fill_(1.0)
        self.grads, self.momentum, self.second = (torch.zeros_like(self.params) for _ in range(3))
        if blocks > 0:
            self.matrices = [self.offset["W2"]] + [(self.offset[f"W{i}"][0] + t * width * width, width, width) for i in range(blocks) for t in range(types)]
            self.type_starts = torch.arange(types + 1, device=dev) * nodes // types
        else:
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

    def _block(self, i: int, p, step: int, train: bool):
        """Arguments of the residual norm that ends block i - 1 and begins block i (i = 0: only the norm before the first)."""
        args = dict(pre_norm="rms", pre=p["pre"][i])
        if i > 0:
            args.update(post_norm="rms", post=p["post"][i - 1], gate=p["gate"][i - 1], p=self.dropout if train else 0.0, seed=self.seed * self.blocks + i, step=step)
        return args

    def forward_blocks(self, ids, step: int = 0, train: bool = False):
        """Output rows of the ids and what the way back needs, all in the order of the sorted ids, whose permutation comes first."""
        t = self.torch
        ids, order = t.sort(ids)
        p = {n: self.part(self.params, n) for n in self.offset}
        offsets = t.searchsorted(ids, self.type_starts).to(t.int32)
        s = self.ctx.embed(p["E"], ids, scale=self.scale)
        s, n = self.ctx.residual_norm(s, dtype=t.bfloat16, **self._block(0, p, step, train))
        kept = []
        for i in range(self.blocks):
            w = p[f"W{i}"].view(self.types, self.width, self.width).to(t.bfloat16)
            h = self.ctx.grouped_linear(n, offsets, w, bias=p[f"b{i}"], relu=True)
            after, n_after = self.ctx.residual_norm(s, h, **self._block(i + 1, p, step, train))
            kept.append((s, n, h, w))
            s, n = after, n_after
        w2 = p["W2"].to(t.bfloat16)
        return order, ids, offsets, kept, s, n, w2, self.ctx.op_linear(n, w2, p["b2"].reshape(-1).contiguous())

    def backward_blocks(self, dz, ids, offsets, kept, s, n, w2, step: int):
        """Gradients of all parameters from that of the (sorted) output rows."""
        t = self.torch
        p, g = ({name: self.part(flat, name) for name in self.offset} for flat in (self.params, self.grads))
        dz16 = dz.to(t.bfloat16)
        g["b2"].copy_(dz.sum(0, keepdim=True))
        g["W2"].copy_(self.ctx.op_weight_grad(n, dz16))
        ds, dn = None, self.ctx.op_linear(dz16, w2, trans_b=True)
        for i in reversed(range(self.blocks)):
            before, n, h, w = kept[i]
            got = self.ctx.residual_norm_grad(ds, dn, s, h, dpre=g["pre"][i + 1], dpost=g["post"][i], dgate=g["gate"][i], **self._block(i + 1, p, step, True))
            ds, dh = got["dx"], got["dh"] * (h > 0)
            self.ctx.grouped_weight_grad(n, dh, offsets, dW=g[f"W{i}"].view(self.types, self.width, self.width), dbias=g[f"b{i}"])
            dn = self.ctx.grouped_linear(dh, offsets, w, trans_b=True)
            s = before
        dx = self.ctx.residual_norm_grad(ds, dn, s, dpre=g["pre"][0], **self._block(0, p, step, True))["dx"]
        self.ctx.embed_grad(dx, ids, self.nodes, scale=self.scale, grad=g["E"])

    def step(self, src, dst, neg, lr: float = 0.02, adam_lr: float = 3e-3) -> float:
        """One update on the edges (src, dst) and the non-edges (src, neg); returns the loss before it."""
        t = self.torch
        B = src.numel()
        ids = t.cat((src, dst, neg))
        if self.blocks > 0:
            order, *state, z = self.forward_blocks(ids, self.t, train=True)
            z = t.empty_like(z).index_copy_(0, order, z)
        else:
            x, h, z, w1, w2 = self.forward(ids)
        zs, zd, zn = (part.float() for part in z.view(3, B, self.out))
        pos, negs = (zs * zd).sum(1), (zs * zn).sum(1)
        loss = (t.nn.functional.softplus(-pos).sum() + t.nn.functional.softplus(negs).sum()) / (2 * B)
        gp, gn = ((t.sigmoid(pos) - 1.0) / (2 * B))[:, None], (t.sigmoid(negs) / (2 * B))[:, None]
        dz = t.cat((gp * zd + gn * zn, gp * zs, gn * zs))
        if self.blocks > 0:
            self.backward_blocks(dz[order], *state, self.t)
        else:
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
    ap.add_argument("--types", type=int, default=1, help="node types, runs of ids, with weight matrices of their own in the residual blocks")
    ap.add_argument("--blocks", type=int, default=0, help="residual blocks in the place of the first transform")
    ap.add_argument("--dropout", type=float, default=0.0, help="of the residual blocks")
    args = ap.parse_args()
    if args.blocks <= 0 and (args.types != 1 or args.dropout != 0.0):
        ap.error("--types and --dropout belong to the residual blocks: give --blocks, too")

    import torch
    import workloads as wl
    from . import Context

    g = wl.chung_lu(args.nodes, args.mean_degree, 2.1, seed=args.seed)
    ctx = Context(0)
    ctx.load_graph(g.n, g.rowptr, g.col, None, wl.node_features(g.n, 8, args.seed))
    u, v = (torch.from_numpy(x).to("cuda:0") for x in wl.undirected_edge_list(g))
    model = LearnedFeatures(ctx, g.n, args.width, seed=args.seed, types=args.types, blocks=args.blocks, dropout=args.dropout)
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
