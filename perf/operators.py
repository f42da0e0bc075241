"""Cases of the learned-feature and matrix-optimiser operators: node embedding lookup with scaling, its gradient by
sorted ids, orthogonalisation of an update by Newton-Schulz products, and the weight update built on it.

`run` computes a case in plain 32-bit torch operations (`own = False`) or through the library (`own = True`);
`exact` gives the same outputs from the definitions in 64 bits.

Definitions
  embed         out[i] = scale * table[ids[i]], 0 where ids[i] is the padding id
  embed_grad    grad[v] = scale * sum of dout[i] over the i with ids[i] = v, 0 for the padding id and rows never named
  orthogonalize X <- X / (|X|_F + 1e-7), then five times X <- a X + (b A + c A^2) X with A = X X^T
                (a, b, c) = (3.4445, -4.7750, 2.0315); matrices with more rows than columns are iterated transposed
  muon_step     weight matrices W [in, out]: M <- mu M + g, u = g + mu M,
                W <- (1 - lr wd) W - lr sqrt(max(1, out / in)) orthogonalize(u); every other parameter: Adam
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
COEFFS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
STEPS = 5
MUON = dict(lr=0.02, mu=0.95, weight_decay=0.01, adam_lr=1e-3, beta1=0.9, beta2=0.999, adam_eps=1e-8, t=3)
NO_PADDING = -(1 << 31)

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
        # a mini-batch of 256 positives on the 2,000-node graph: source, destination and one negative each
        dict(name="embed_batch256", op="embed", rows=2000, width=64, tokens=768, table="fp32", out="fp32", padding=False),
        # a full batch of 65,536 positives on the million-node graph; FP32 master table, BF16 rows for the transforms
        dict(name="embed_batch65536", op="embed", rows=1_000_000, width=256, tokens=196_608, table="fp32", out="bf16", padding=False),
        # the gradient of the small mini-batch
        dict(name="grad_batch256", op="embed_grad", rows=2000, width=64, tokens=768, dout="fp32", grad="fp32", padding=False),
        # a ragged batch on the co-author graph, an odd number of ids, some of them padding, width 100
        dict(name="grad_ragged", op="embed_grad", rows=235_000, width=100, tokens=200_001, dout="fp32", grad="fp32", padding=True),
        # the outermost frontier of a sampled step on the citation graph: 2.9 M rows, about two million ids
        dict(name="grad_frontier", op="embed_grad", rows=2_900_000, width=128, tokens=1_966_080, dout="bf16", grad="fp32", padding=False),
        # one weight matrix of the smallest encoder: latency alone
        dict(name="orth_64", op="orthogonalize", batch=1, rows=64, cols=64, dtype="fp32"),
        # the stacked weights of many emulated workers at once, tall
        dict(name="orth_workers", op="orthogonalize", batch=16, rows=512, cols=256, dtype="bf16"),
        # an odd shape in FP32
        dict(name="orth_ragged", op="orthogonalize", batch=1, rows=1000, cols=417, dtype="fp32"),
        # a large square update in BF16
        dict(name="orth_4096", op="orthogonalize", batch=1, rows=4096, cols=4096, dtype="bf16"),
        # the encoder of the benchmark: two-layer SAGE 128-256-256
        dict(name="muon_sage2", op="muon_step", arch="sage", d0=128, d1=256, d2=256, d3=0, pred=0),
        # three-layer SAGE 128-256-256-256 with the MLP predictor of width 256
        dict(name="muon_sage3_mlp", op="muon_step", arch="sage", d0=128, d1=256, d2=256, d3=256, pred=256),
        # a wide encoder of odd widths
        dict(name="muon_wide", op="muon_step", arch="gcn", d0=1000, d1=1999, d2=1500, d3=417, pred=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A width of the range: half of them multiples of 64, the others any number."""
    w = _log_int(rng, lo, hi)
    return max(64, w // 64 * 64) if rng.random() < 0.5 and w >= 64 else w


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "embed_grad", "orthogonalize", "orthogonalize", "muon_step"])
    if op in ("embed", "embed_grad"):
        rows, tokens, width = _log_int(rng, 500, 2_900_000), _log_int(rng, 100, 1_966_080), _width(rng, 16, 512)
        if op == "embed":
            tokens = min(tokens, max(100, 50_000_000 // width))
            table, out = rng.choice([("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16")])
            rows = min(rows, 256_000_000 // width)
            return dict(op=op, rows=rows, width=width, tokens=tokens, table=table, out=out, padding=rng.random() < 0.3)
        rows = min(rows, max(500, 300_000_000 // width))
        tokens = min(tokens, max(100, 200_000_000 // width))
        dout, grad = rng.choice([("fp32", "fp32"), ("bf16", "fp32"), ("bf16", "bf16")])
        return dict(op=op, rows=rows, width=width, tokens=tokens, dout=dout, grad=grad, padding=rng.random() < 0.3)
    if op == "orthogonalize":
        rows, cols = _width(rng, 32, 2048), _width(rng, 32, 2048)
        batch = min(_log_int(rng, 1, 32), max(1, 4_000_000 // (rows * cols)))
        return dict(op=op, batch=batch, rows=rows, cols=cols, dtype=rng.choice(["fp32", "bf16"]))
    arch = rng.choice(["sage", "gcn"])
    d = [_width(rng, 64, 1024) for _ in range(4)]
    if rng.random() < 0.5:
        d[3] = 0
    return dict(op=op, arch=arch, d0=d[0], d1=d[1], d2=d[2], d3=d[3], pred=rng.choice([0, 0, 256]))


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1_000_003 + 17)


def _ids(case, gen):
    """Ids as a batch names nodes: two thirds endpoints of edges of a power-law graph (exponent 2.1, shuffled ids), one
    third uniform negatives, and for padded cases about 3 % padding."""
    v, n = case["rows"], case["tokens"]
    weight = torch.arange(v, device="cuda", dtype=torch.float64).add_(10.0).pow_(-1.0 / 1.1)
    cum = weight.cumsum(0)
    rank = torch.searchsorted(cum, torch.rand(n, device="cuda", dtype=torch.float64, generator=gen) * cum[-1]).clamp_(max=v - 1)
    ids = torch.randperm(v, device="cuda", generator=gen)[rank]
    uniform = torch.randint(0, v, (n,), device="cuda", generator=gen)
    kind = torch.rand(n, device="cuda", generator=gen)
    ids = torch.where(kind < 1.0 / 3.0, uniform, ids)
    if case["padding"]:
        ids = torch.where(torch.rand(n, device="cuda", generator=gen) < 0.03, -1, ids)
    return ids.to(torch.int32)


def _update(shape, gen):
    """A gradient-like matrix: a decaying spectrum (a few strong directions) over noise."""
    rows, cols = shape[-2:]
    r = min(16, rows, cols)
    lead = shape[:-2]
    left = torch.randn(*lead, rows, r, device="cuda", generator=gen)
    right = torch.randn(*lead, r, cols, device="cuda", generator=gen)
    strength = 0.5 ** torch.arange(r, device="cuda", dtype=torch.float32)
    return 1e-3 * (torch.randn(*shape, device="cuda", generator=gen) + (left * strength) @ right)


def _layout(case):
    """(offset, rows, cols) of every weight matrix and the length of the flat parameter vector: per layer its matrices and
    its bias, then the MLP predictor's W0, b0, W1, b1, w2, b2."""
    dims = [d for d in (case["d0"], case["d1"], case["d2"], case["d3"]) if d]
    mats, at = [], 0
    for fi, fo in zip(dims[:-1], dims[1:]):
        for _ in range(2 if case["arch"] == "sage" else 1):
            mats.append((at, fi, fo))
            at += fi * fo
        at += fo
    if case["pred"]:
        h = case["pred"]
        for fi in (dims[-1], h):
            mats.append((at, fi, h))
            at += fi * h + h
        at += h + 1
    return mats, at


def prepare(case, seed):
    gen = _generator(seed)
    state = {"case": case}
    op = case["op"]
    if op == "embed":
        state["ids"] = _ids(case, gen)
        state["table"] = torch.randn(case["rows"], case["width"], device="cuda", generator=gen).mul_(0.1).to(DTYPES[case["table"]])
        state["scale"] = math.sqrt(case["width"])
    elif op == "embed_grad":
        state["ids"] = _ids(case, gen)
        state["dout"] = torch.randn(case["tokens"], case["width"], device="cuda", generator=gen).mul_(1e-3).to(DTYPES[case["dout"]])
        state["scale"] = math.sqrt(case["width"])
    elif op == "orthogonalize":
        state["x"] = _update((case["batch"], case["rows"], case["cols"]), gen).to(DTYPES[case["dtype"]])
    else:
        mats, n = _layout(case)
        params = torch.randn(n, device="cuda", generator=gen).mul_(0.05)
        grads = torch.randn(n, device="cuda", generator=gen).mul_(1e-3)
        momentum = torch.randn(n, device="cuda", generator=gen).mul_(1e-3)
        for at, r, c in mats:
            grads[at:at + r * c] = _update((r, c), gen).reshape(-1)
            momentum[at:at + r * c] = 5.0 * _update((r, c), gen).reshape(-1)
        vector = torch.ones(n, dtype=torch.bool, device="cuda")
        for at, r, c in mats:
            vector[at:at + r * c] = False
        state.update(params=params, grads=grads, momentum=momentum, adam_v=grads.square().mul_(0.5), matrices=mats,
                     vector=vector.nonzero().reshape(-1))
    return state


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_embed(s):
    case, ids = s["case"], s["ids"].long()
    out = s["table"][ids.clamp(min=0)].float() * s["scale"]
    if case["padding"]:
        out = torch.where((ids >= 0)[:, None], out, 0.0)
    return out.to(DTYPES[case["out"]])


def _plain_embed_grad(s):
    case, ids = s["case"], s["ids"].long()
    rows = s["dout"].float() * s["scale"]
    if case["padding"]:
        rows = torch.where((ids >= 0)[:, None], rows, 0.0)
    grad = torch.zeros(case["rows"], case["width"], device="cuda")
    grad.index_add_(0, ids.clamp(min=0), rows)
    return grad.to(DTYPES[case["grad"]])


def _plain_orthogonalize(x):
    tall = x.shape[-2] > x.shape[-1]
    x = x.float()
    if tall:
        x = x.mT
    x = x / (x.square().sum(dim=(-2, -1), keepdim=True).sqrt() + EPS)
    a, b, c = COEFFS
    for _ in range(STEPS):
        gram = x @ x.mT
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.mT if tall else x


def _plain_muon(s):
    m, g, p = MUON, s["grads"], s["params"]
    momentum = m["mu"] * s["momentum"] + g
    new = p.clone()
    update = g + m["mu"] * momentum
    for at, r, c in s["matrices"]:
        o = _plain_orthogonalize(update[at:at + r * c].view(r, c))
        new[at:at + r * c] = (1 - m["lr"] * m["weight_decay"]) * p[at:at + r * c] - m["lr"] * math.sqrt(max(1.0, c / r)) * o.reshape(-1)
    i = s["vector"]
    v = s["adam_v"].clone()
    momentum[i] = m["beta1"] * s["momentum"][i] + (1 - m["beta1"]) * g[i]
    v[i] = m["beta2"] * v[i] + (1 - m["beta2"]) * g[i].square()
    c1, c2 = 1 - m["beta1"] ** m["t"], 1 - m["beta2"] ** m["t"]
    new[i] = p[i] - m["adam_lr"] * (momentum[i] / c1) / ((v[i] / c2).sqrt() + m["adam_eps"])
    return new, momentum, v


def run(state):
    case, op = state["case"], state["case"]["op"]
    if own:
        ctx = _ctx()
        if op == "embed":
            return ctx.embed(state["table"], state["ids"], scale=state["scale"], padding_id=-1 if case["padding"] else None, out_dtype=DTYPES[case["out"]])
        if op == "embed_grad":
            return ctx.embed_grad(state["dout"], state["ids"], case["rows"], scale=state["scale"], padding_id=-1 if case["padding"] else None,
                                  grad_dtype=DTYPES[case["grad"]])
        if op == "orthogonalize":
            return ctx.orthogonalize(state["x"], steps=STEPS, coeffs=COEFFS, eps=EPS)
        out = tuple(torch.empty_like(state[k]) for k in ("params", "momentum", "adam_v"))
        return ctx.muon_step(state["params"], state["momentum"], state["adam_v"], state["grads"], t=MUON["t"], matrices=state["matrices"], lr=MUON["lr"],
                             mu=MUON["mu"], weight_decay=MUON["weight_decay"], adam_lr=MUON["adam_lr"], beta1=MUON["beta1"], beta2=MUON["beta2"],
                             adam_eps=MUON["adam_eps"], steps=STEPS, coeffs=COEFFS, ns_eps=EPS, out=out)
    if op == "embed":
        return _plain_embed(state)
    if op == "embed_grad":
        return _plain_embed_grad(state)
    if op == "orthogonalize":
        return _plain_orthogonalize(state["x"]).to(state["x"].dtype)
    return _plain_muon(state)


# ------------------------------------------------------------------------------------------------ work
def _ns_flops(r, c):
    m, n = min(r, c), max(r, c)
    return STEPS * (3.0 * m * m * n + 1.0 * m * m * m)  # the two symmetric products count their upper triangles


def work(case):
    size = {"fp32": 4, "bf16": 2}
    op = case["op"]
    if op == "embed":
        # every id, every distinct row once (an expectation is not needed: at most one row per id or per table row), every output row
        n, d = case["tokens"], case["width"]
        return {"bytes": 4.0 * n + min(n, case["rows"]) * d * size[case["table"]] + n * d * size[case["out"]], "flops": 1.0 * n * d}
    if op == "embed_grad":
        n, d = case["tokens"], case["width"]
        return {"bytes": 4.0 * n + n * d * size[case["dout"]] + case["rows"] * d * size[case["grad"]], "flops": 1.0 * n * d}
    if op == "orthogonalize":
        elems = case["batch"] * case["rows"] * case["cols"]
        return {"bytes": 2.0 * elems * size[case["dtype"]], "flops": case["batch"] * _ns_flops(case["rows"], case["cols"])}
    mats, n = _layout(case)
    inside = sum(r * c for _, r, c in mats)
    # matrices: weights, momentum and gradient read, weights and momentum written; the rest: Adam's seven arrays
    return {"bytes": 4.0 * (5 * inside + 7 * (n - inside)), "flops": sum(_ns_flops(r, c) for _, r, c in mats) + 10.0 * n}


# ------------------------------------------------------------------------------------------------ 64 bits
def _exact_orthogonalize(x):
    """The same map written on the other side: x p(x^T x), with the Gram matrix of the narrow side kept separate."""
    x = x.double()
    a, b, c = COEFFS
    y = x / (torch.linalg.matrix_norm(x, keepdim=True) + EPS)
    for _ in range(STEPS):
        if y.shape[-2] >= y.shape[-1]:
            g = torch.einsum("...ki,...kj->...ij", y, y)
            poly = b * g + c * torch.linalg.matrix_power(g, 2)
            poly.diagonal(dim1=-2, dim2=-1).add_(a)
            y = y @ poly
        else:
            g = torch.einsum("...ik,...jk->...ij", y, y)
            poly = b * g + c * torch.linalg.matrix_power(g, 2)
            poly.diagonal(dim1=-2, dim2=-1).add_(a)
            y = poly @ y
    return y


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        keep = (s["ids"] >= 0).double()
        return torch.index_select(s["table"], 0, s["ids"].clamp(min=0)).double() * (keep * s["scale"])[:, None]
    if op == "embed_grad":
        # sorted ids, running sums inside each run of equal ids, taken at the ends of the runs
        order = torch.argsort(s["ids"], stable=True)
        ids, rows = s["ids"][order].long(), s["dout"][order].double()
        named, count = torch.unique_consecutive(ids, return_counts=True)
        sums = torch.segment_reduce(rows, "sum", lengths=count, axis=0)
        grad = torch.zeros(case["rows"], case["width"], dtype=torch.float64, device="cuda")
        real = named >= 0
        grad[named[real]] = sums[real] * s["scale"]
        return grad
    if op == "orthogonalize":
        return _exact_orthogonalize(s["x"])
    m = MUON
    g, p, v = s["grads"].double(), s["params"].double(), s["adam_v"].double()
    b1, b2 = m["beta1"], m["beta2"]
    moment = b1 * s["momentum"].double() + (1 - b1) * g
    second = b2 * v + (1 - b2) * g * g
    step = moment / (1 - b1 ** m["t"]) / (torch.sqrt(second / (1 - b2 ** m["t"])) + m["adam_eps"])
    new = p - m["adam_lr"] * step
    for at, r, c in s["matrices"]:
        span = slice(at, at + r * c)
        moment[span] = m["mu"] * s["momentum"][span].double() + g[span]
        second[span] = v[span]
        o = _exact_orthogonalize((g[span] + m["mu"] * moment[span]).reshape(r, c))
        new[span] = p[span] - m["lr"] * (m["weight_decay"] * p[span] + math.sqrt(max(1.0, c / r)) * o.reshape(-1))
    return new, moment, second
