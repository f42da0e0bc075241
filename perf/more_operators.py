"""Cases of the residual-block operators for typed nodes: dropout from a counter-based generator, the norms around a block
fused with its dropout, gate and residual sum, products with one weight matrix per group of rows, and their gradients.

`run` computes a case in plain 32-bit torch operations (`own = False`) or through the library (`own = True`);
`exact` gives the same outputs from the definitions in 64 bits.

Definitions
  dropout              out = in * 65536 / (65536 - t) where u >= t, else 0; t = round(65536 p); u is the 16-bit half c % 2 of word
                       (c % 8) / 2 of Philox4x32-10 with counter (row, row >> 32, step, 5 | (c / 8) << 8) and key = seed
  residual_norm        y = x + scale * gate * dropout(post(h)), n = pre(y); post, pre: RMS or layer norm with weight (and bias)
  residual_norm_grad   gradients of x, h, gate and the norms' parameters from those of y and n
  grouped_linear       rows offsets[g] .. offsets[g + 1] - 1: C = act(A B[g] + bias[g]), or A B[g]^T (the input gradient)
  grouped_weight_grad  dW[g] = A^T dZ and dbias[g] = column sums of dZ over the rows of group g
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6
SCALE = 0.5
STEP = 11
MASK32 = 0xFFFFFFFF

_context = None


def _ctx():
    """The library context, kept for the life of the process as a training program does."""
    global _context
    if _context is None:
        import paper_2506_20818_b200 as pkg
        _context = pkg.Context(0)
    return _context


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # rows of a mini-batch of 256 positives: source, destination and one negative each; latency alone
        dict(name="dropout_batch256", op="dropout", rows=768, width=64, dtype="fp32", p=0.5),
        # activations of the million-node graph
        dict(name="dropout_nodes", op="dropout", rows=1_000_000, width=256, dtype="bf16", p=0.1),
        # between two blocks, the small mini-batch
        dict(name="block_batch256", op="residual_norm", rows=768, width=64, stream="fp32", dtype="fp32", norm="rms", post=True, bias=False,
             gate="vector", p=0.0),
        # a full batch of 65,536 positives, FP32 residual sum beside BF16 blocks, norm after the block, dropout, learned column gate
        dict(name="block_batch65536", op="residual_norm", rows=196_608, width=256, stream="fp32", dtype="bf16", norm="rms", post=True, bias=False,
             gate="vector", p=0.1),
        # its gradient
        dict(name="block_grad_batch65536", op="residual_norm_grad", rows=196_608, width=256, stream="fp32", dtype="bf16", norm="rms", post=True,
             bias=False, gate="vector", p=0.1),
        # an odd number of rows and an odd width, layer norms with biases, a gate per element
        dict(name="block_grad_ragged", op="residual_norm_grad", rows=50_001, width=417, stream="fp32", dtype="fp32", norm="layer", post=True, bias=True,
             gate="matrix", p=0.2),
        # the small mini-batch over four node types
        dict(name="grouped_batch256", op="grouped_linear", rows=768, k=64, n=64, groups=4, dtype="fp32", trans=False, act=True),
        # a full batch over eight partitions, benchmark width
        dict(name="grouped_batch65536", op="grouped_linear", rows=196_608, k=256, n=256, groups=8, dtype="bf16", trans=False, act=True),
        # the input gradient of a wide transform of odd widths, forty types, some without a row
        dict(name="grouped_ragged", op="grouped_linear", rows=30_011, k=1999, n=1000, groups=40, dtype="bf16", trans=True, act=False),
        # one FP32 layer of the co-author graph by sixteen types
        dict(name="grouped_fp32", op="grouped_linear", rows=100_003, k=256, n=512, groups=16, dtype="fp32", trans=False, act=True),
        # weight gradients: the full batch in BF16, and FP32 of odd widths
        dict(name="grouped_wgrad_batch65536", op="grouped_weight_grad", rows=196_608, k=256, n=256, groups=8, dtype="bf16"),
        dict(name="grouped_wgrad_ragged", op="grouped_weight_grad", rows=30_011, k=417, n=1000, groups=40, dtype="fp32"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A width of the range: half of them multiples of 64, the others any number."""
    w = _log_int(rng, lo, hi)
    return max(64, w // 64 * 64) if rng.random() < 0.5 and w >= 64 else w


def draw(rng):
    op = rng.choice(["dropout", "residual_norm", "residual_norm_grad", "grouped_linear", "grouped_linear", "grouped_weight_grad"])
    if op == "dropout":
        width = _width(rng, 16, 2048)
        return dict(op=op, rows=min(_log_int(rng, 100, 1_000_000), 250_000_000 // width), width=width, dtype=rng.choice(["fp32", "bf16"]),
                    p=rng.choice([0.1, 0.2, 0.5]))
    if op in ("residual_norm", "residual_norm_grad"):
        width = _width(rng, 16, 2048)
        stream, dtype = rng.choice([("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16")])
        norm = rng.choice(["rms", "layer"])
        return dict(op=op, rows=min(_log_int(rng, 100, 400_000), 50_000_000 // width), width=width, stream=stream, dtype=dtype, norm=norm,
                    post=rng.random() < 0.6, bias=norm == "layer", gate=rng.choice(["none", "vector", "matrix"]), p=rng.choice([0.0, 0.1, 0.5]))
    k, n = _width(rng, 16, 2048), _width(rng, 16, 2048)
    rows = min(_log_int(rng, 100, 400_000), 60_000_000_000 // (k * n))
    groups = min(_log_int(rng, 1, 200), max(1, 200_000_000 // (k * n)))
    case = dict(op=op, rows=rows, k=k, n=n, groups=groups, dtype=rng.choice(["fp32", "bf16"]))
    if op == "grouped_linear":
        case["trans"] = rng.random() < 0.4
        case["act"] = not case["trans"]
    return case


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1_000_003 + 29)


def _randn(gen, *shape, scale=1.0, dtype=torch.float32):
    return torch.randn(*shape, device="cuda", generator=gen).mul_(scale).to(dtype)


def _offsets(case, gen):
    """Sizes of the groups follow a power law in shuffled order, one in eight has no row; they cover all rows."""
    g = case["groups"]
    weight = torch.arange(1, g + 1, device="cuda", dtype=torch.float64).pow_(-0.7)[torch.randperm(g, device="cuda", generator=gen)]
    if g >= 4:
        weight[torch.randperm(g, device="cuda", generator=gen)[:g // 8]] = 0.0
    ends = (weight.cumsum(0) / weight.sum() * case["rows"]).round_().to(torch.int32).clamp_(max=case["rows"])
    ends[-1] = case["rows"]
    return torch.cat((torch.zeros(1, dtype=torch.int32, device="cuda"), ends))


def prepare(case, seed):
    gen = _generator(seed)
    op = case["op"]
    s = {"case": case, "seed": int(seed) * 7919 + 1}
    if op == "dropout":
        s["x"] = _randn(gen, case["rows"], case["width"], dtype=DTYPES[case["dtype"]])
    elif op in ("residual_norm", "residual_norm_grad"):
        r, d = case["rows"], case["width"]
        stream, dtype = DTYPES[case["stream"]], DTYPES[case["dtype"]]
        s["h"] = _randn(gen, r, d, scale=0.7, dtype=dtype)
        s["pre"] = 1.0 + _randn(gen, d, scale=0.1)
        s["post"] = 1.0 + _randn(gen, d, scale=0.1) if case["post"] else None
        s["pre_bias"] = _randn(gen, d, scale=0.1) if case["bias"] else None
        s["post_bias"] = _randn(gen, d, scale=0.1) if case["bias"] and case["post"] else None
        s["gate"] = None
        if case["gate"] == "vector":
            s["gate"] = 1.0 + _randn(gen, d, scale=0.2)
        elif case["gate"] == "matrix":
            s["gate"] = torch.sigmoid(_randn(gen, r, d)).to(dtype)
        if op == "residual_norm":
            s["x"] = _randn(gen, r, d, scale=1.5, dtype=stream)
        else:
            s["y"] = _randn(gen, r, d, scale=1.6, dtype=stream)
            s["dy"] = _randn(gen, r, d, scale=1e-3, dtype=stream)
            s["dn"] = _randn(gen, r, d, scale=1e-3, dtype=dtype)
    else:
        r, k, n, g = case["rows"], case["k"], case["n"], case["groups"]
        dtype = DTYPES[case["dtype"]]
        s["offsets"] = _offsets(case, gen)
        s["bounds"] = s["offsets"].tolist()  # the plain form walks the groups on the host
        s["a"] = _randn(gen, r, k, dtype=dtype)
        if op == "grouped_linear":
            s["b"] = _randn(gen, g, n, k, scale=1.0 / math.sqrt(k), dtype=dtype) if case["trans"] else _randn(gen, g, k, n, scale=1.0 / math.sqrt(k), dtype=dtype)
            s["bias"] = _randn(gen, g, n, scale=0.05) if case["act"] else None
        else:
            s["dz"] = _randn(gen, r, n, scale=1e-3, dtype=dtype)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_keep(rows, width, p, seed):
    """Boolean [rows, width]: which elements stay, and the factor on them."""
    blocks = (width + 7) // 8
    t = int(round(65536.0 * p))
    row = torch.arange(rows, device="cuda", dtype=torch.int64)[:, None].expand(rows, blocks)
    c0, c1, c2 = row & MASK32, row >> 32, torch.full_like(row, STEP & MASK32)
    c3 = (5 | torch.arange(blocks, device="cuda", dtype=torch.int64) << 8)[None, :].expand(rows, blocks)
    k0, k1 = seed & MASK32, (seed >> 32) & MASK32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & MASK32) ^ c1 ^ k0, p1 & MASK32, ((p0 >> 32) & MASK32) ^ c3 ^ k1, p0 & MASK32
        k0, k1 = (k0 + 0x9E3779B9) & MASK32, (k1 + 0xBB67AE85) & MASK32
    halves = torch.stack([h for w in (c0, c1, c2, c3) for h in (w & 0xFFFF, w >> 16)], dim=-1).reshape(rows, blocks * 8)
    return halves[:, :width] >= t, 65536.0 / (65536 - t)


def _plain_norm(x, kind, weight, bias):
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    x = x / (x.square().mean(1, keepdim=True) + EPS).sqrt()
    x = x * weight
    return x if bias is None else x + bias


def _plain_norm_grad(x, kind, weight, dout):
    """Gradients of x, the weight and the bias."""
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    r = 1.0 / (x.square().mean(1, keepdim=True) + EPS).sqrt()
    hat, u = x * r, dout * weight
    dx = u - hat * (u * hat).mean(1, keepdim=True)
    if kind == "layer":
        dx = dx - u.mean(1, keepdim=True)
    return dx * r, (dout * hat).sum(0), dout.sum(0)


def _plain_residual(s):
    case = s["case"]
    b = s["h"].float()
    if case["post"]:
        b = _plain_norm(b, case["norm"], s["post"], s["post_bias"])
    if case["p"] > 0:
        keep, factor = _plain_keep(case["rows"], case["width"], case["p"], s["seed"])
        b = torch.where(keep, b * factor, 0.0)
    if s["gate"] is not None:
        b = b * s["gate"].float()
    y = s["x"].float() + SCALE * b
    return y.to(s["x"].dtype), _plain_norm(y, case["norm"], s["pre"], s["pre_bias"]).to(s["h"].dtype)


def _plain_residual_grad(s):
    case = s["case"]
    g, dpre, dpre_bias = _plain_norm_grad(s["y"].float(), case["norm"], s["pre"], s["dn"].float())
    g = g + s["dy"].float()
    h = s["h"].float()
    b = _plain_norm(h, case["norm"], s["post"], s["post_bias"]) if case["post"] else h
    keep = None
    if case["p"] > 0:
        keep, factor = _plain_keep(case["rows"], case["width"], case["p"], s["seed"])
        b = torch.where(keep, b * factor, 0.0)
    db, dgate = SCALE * g, None
    if s["gate"] is not None:
        dgate = db * b
        dgate = dgate.sum(0) if case["gate"] == "vector" else dgate.to(s["gate"].dtype)
        db = db * s["gate"].float()
    if keep is not None:
        db = torch.where(keep, db * factor, 0.0)
    dpost = dpost_bias = None
    if case["post"]:
        db, dpost, dpost_bias = _plain_norm_grad(h, case["norm"], s["post"], db)
    return _grads(case, g.to(s["dy"].dtype), db.to(s["h"].dtype), dgate, dpre, dpre_bias, dpost, dpost_bias)


def _grads(case, dx, dh, dgate, dpre, dpre_bias, dpost, dpost_bias):
    """The gradients that the case has."""
    out = {"dx": dx, "dh": dh, "dpre": dpre}
    if case["gate"] != "none":
        out["dgate"] = dgate
    if case["post"]:
        out["dpost"] = dpost
    if case["bias"]:
        out["dpre_bias"] = dpre_bias
        if case["post"]:
            out["dpost_bias"] = dpost_bias
    return out


def _plain_grouped(s):
    case = s["case"]
    out = torch.zeros(case["rows"], case["n"], dtype=s["a"].dtype, device="cuda")
    for g, (lo, hi) in enumerate(zip(s["bounds"][:-1], s["bounds"][1:])):
        if hi > lo:
            w = s["b"][g].float()
            c = s["a"][lo:hi].float() @ (w.T if case["trans"] else w)
            if case["act"]:
                c = torch.clamp(c + s["bias"][g], min=0.0)
            out[lo:hi] = c.to(out.dtype)
    return out


def _plain_grouped_grad(s):
    case = s["case"]
    dw = torch.zeros(case["groups"], case["k"], case["n"], device="cuda")
    db = torch.zeros(case["groups"], case["n"], device="cuda")
    for g, (lo, hi) in enumerate(zip(s["bounds"][:-1], s["bounds"][1:])):
        if hi > lo:
            dz = s["dz"][lo:hi].float()
            dw[g] = s["a"][lo:hi].float().T @ dz
            db[g] = dz.sum(0)
    return dw, db


def run(state):
    s, case = state, state["case"]
    op = case["op"]
    if own:
        ctx = _ctx()
        if op == "dropout":
            return ctx.dropout(s["x"], case["p"], seed=s["seed"], step=STEP)
        if op == "grouped_linear":
            return ctx.grouped_linear(s["a"], s["offsets"], s["b"], bias=s["bias"], relu=case["act"], trans_b=case["trans"])
        if op == "grouped_weight_grad":
            return ctx.grouped_weight_grad(s["a"], s["dz"], s["offsets"], bias=True)
        block = dict(pre_norm=case["norm"], pre=s["pre"], pre_bias=s["pre_bias"], post_norm=case["norm"] if case["post"] else None, post=s["post"],
                     post_bias=s["post_bias"], gate=s["gate"], scale=SCALE, p=case["p"], seed=s["seed"], step=STEP, eps=EPS)
        if op == "residual_norm":
            return ctx.residual_norm(s["x"], s["h"], **block)
        got = ctx.residual_norm_grad(s["dy"], s["dn"], s["y"], s["h"], **block)
        return _grads(case, got["dx"], got["dh"], got.get("dgate"), got["dpre"], got.get("dpre_bias"), got.get("dpost"), got.get("dpost_bias"))
    if op == "dropout":
        keep, factor = _plain_keep(case["rows"], case["width"], case["p"], s["seed"])
        return torch.where(keep, s["x"].float() * factor, 0.0).to(s["x"].dtype)
    if op == "residual_norm":
        return _plain_residual(s)
    if op == "residual_norm_grad":
        return _plain_residual_grad(s)
    return _plain_grouped(s) if op == "grouped_linear" else _plain_grouped_grad(s)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    size = {"fp32": 4.0, "bf16": 2.0}
    op = case["op"]
    if op == "dropout":
        return {"bytes": 2 * size[case["dtype"]] * case["rows"] * case["width"], "flops": 1.0 * case["rows"] * case["width"]}
    if op in ("residual_norm", "residual_norm_grad"):
        e = 1.0 * case["rows"] * case["width"]
        a, b = size[case["stream"]], size[case["dtype"]]
        gate = b if case["gate"] == "matrix" else 0.0
        if op == "residual_norm":  # x, h in, y, n out
            return {"bytes": e * (2 * a + 2 * b + gate), "flops": 12 * e}
        return {"bytes": e * (3 * a + 3 * b + 2 * gate), "flops": 30 * e}  # dy, y, dn, h in, dx, dh out
    r, k, n, g, b = case["rows"], case["k"], case["n"], case["groups"], size[case["dtype"]]
    flops = 2.0 * r * k * n
    if op == "grouped_linear":
        return {"bytes": b * (1.0 * r * k + 1.0 * r * n + 1.0 * g * k * n), "flops": flops}
    return {"bytes": b * (1.0 * r * k + 1.0 * r * n) + 4.0 * g * n * (k + 1.0), "flops": flops}


# ------------------------------------------------------------------------------------------------ 64 bits
def _exact_keep(case, seed):
    """The mask with the generator's products taken from 16-bit limbs, every word on its own."""
    rows, width = case["rows"], case["width"]

    def mul(a, m):  # high and low word of a * m
        low, high = (a & 0xFFFF) * m, (a >> 16) * m
        mid = high + (low >> 16)
        return mid >> 16, ((mid & 0xFFFF) << 16) | (low & 0xFFFF)

    cols = torch.arange((width + 7) // 8, dtype=torch.int64, device="cuda")
    x = torch.arange(rows, dtype=torch.int64, device="cuda")[:, None] + 0 * cols
    ctr = [x % (1 << 32), x // (1 << 32), torch.zeros_like(x) + STEP, torch.zeros_like(x) + 5 + 256 * cols]
    for r in range(10):
        ka, kb = (seed + r * 0x9E3779B9) % (1 << 32), ((seed >> 32) + r * 0xBB67AE85) % (1 << 32)
        (ha, la), (hb, lb) = mul(ctr[0], 0xD2511F53), mul(ctr[2], 0xCD9E8D57)
        ctr = [hb ^ ctr[1] ^ ka, lb, ha ^ ctr[3] ^ kb, la]
    c = torch.arange(width, device="cuda")
    threshold = round(case["p"] * 65536)
    keep = torch.empty(rows, width, dtype=torch.bool, device="cuda")
    for e in range(8):
        word = ctr[e // 2]
        piece = word % 65536 if e % 2 == 0 else word // 65536
        keep[:, c[c % 8 == e]] = piece[:, : int((c % 8 == e).sum())] >= threshold
    return keep.double() * (65536.0 / (65536.0 - threshold))


def _exact_norm(x, kind, weight, bias):
    if kind == "layer":
        out = (x - x.mean(1, keepdim=True)) * torch.rsqrt(x.var(1, unbiased=False, keepdim=True) + EPS)
    else:
        out = x * torch.rsqrt((x * x).sum(1, keepdim=True) / x.shape[1] + EPS)
    return out * weight + (bias if bias is not None else 0.0)


def _exact_branch(case, keep, h, post, post_bias, gate):
    out = _exact_norm(h, case["norm"], post, post_bias) if case["post"] else h
    out = out * keep if keep is not None else out
    return SCALE * (out * gate if gate is not None else out)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "dropout":
        return s["x"].double() * _exact_keep(case, s["seed"])
    if op in ("residual_norm", "residual_norm_grad"):
        d = {k: v.double() if torch.is_tensor(v) else None for k, v in s.items() if k not in ("case", "seed")}
        keep = _exact_keep(case, s["seed"]) if case["p"] > 0 else None
        if op == "residual_norm":
            y = d["x"] + _exact_branch(case, keep, d["h"], d["post"], d["post_bias"], d["gate"])
            return y, _exact_norm(y, case["norm"], d["pre"], d["pre_bias"])
        for k in ("y", "h", "pre", "pre_bias", "post", "post_bias", "gate"):
            if d[k] is not None:
                d[k].requires_grad_(True)
        with torch.enable_grad():
            n = _exact_norm(d["y"], case["norm"], d["pre"], d["pre_bias"])
            n.backward(d["dn"])
            g = d["dy"] + d["y"].grad
            _exact_branch(case, keep, d["h"], d["post"], d["post_bias"], d["gate"]).backward(g)
        grad = {k: d[k].grad if d[k] is not None else None for k in ("h", "pre", "pre_bias", "post", "post_bias", "gate")}
        return _grads(case, g, grad["h"], grad["gate"], grad["pre"], grad["pre_bias"], grad["post"], grad["post_bias"])
    bounds = s["bounds"]
    sizes = [hi - lo for lo, hi in zip(bounds[:-1], bounds[1:])]
    if op == "grouped_linear":
        parts = []
        for g, a in enumerate(torch.split(s["a"], sizes)):
            c = torch.einsum("rk,nk->rn" if case["trans"] else "rk,kn->rn", a.double(), s["b"][g].double())
            parts.append(torch.relu(c + s["bias"][g].double()) if case["act"] else c)
        return torch.cat(parts)
    pairs = list(zip(torch.split(s["a"], sizes), torch.split(s["dz"], sizes)))
    return (torch.stack([torch.einsum("rk,rn->kn", a.double(), z.double()) for a, z in pairs]),
            torch.stack([z.double().sum(0) for _, z in pairs]))
