"""Embedding lookup, its gradient, Newton-Schulz orthogonalisation and the update built on it, against plain 64-bit forms.

Tolerances, derived from the arithmetic:
  lookup          one FP32 product, one rounding: bit for bit what the same two operations give
  gradient        FP32 sums of k terms in any order differ from the exact sum by at most (k + 2) 2^-24 sum |terms| (the 2: the
                  product with the scale and, when accumulating, the addition); a BF16 result is rounded once more, 2^-8 relative
  orthogonalise   every step stores X, A and B with relative errors of 2^-22 (FP32: pairs of FP16) or, in the products, 2^-11
                  (BF16), accumulates with 2^-22 per addition, and an error made in one step is at most about doubled by each
                  later one in directions that are already large (the slope of the polynomial there is at most 1.6 in
                  magnitude).  Five steps: 3 * 2^-22 * (1 + 2 + 4 + 8 + 16) = 2.2e-5 if nothing averaged out; errors are
                  independent, so 2e-5 is demanded for FP32 and, with 2^-12 random instead of 2^-11 and the BF16 rounding of the
                  result (2^-9 at most), 1e-2 for BF16 (relative, Frobenius norm)
  update          lr times the error of the orthogonalisation and a few FP32 roundings of the weight itself: 1e-6 relative
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F64 = torch.float32, torch.bfloat16, torch.float64
COEFFS = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def pkg():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__ as ge
    ge.build()
    import paper_2506_20818_b200 as p
    return p


@pytest.fixture(scope="module")
def ctx(pkg):
    c = pkg.Context(0)
    yield c
    c.close()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def padded(x, extra, offset=0):
    """x on the GPU as a view with `extra` more elements per row, beginning `offset` elements into its storage."""
    rows, cols = x.shape
    buf = torch.full((rows * (cols + extra) + offset + 8,), float("nan"), dtype=x.dtype, device=DEV)
    v = buf[offset:offset + rows * (cols + extra)].view(rows, cols + extra)[:, :cols]
    v.copy_(x)
    return v


# ------------------------------------------------------------------------------------------ lookup
SHAPES = [(1, 1, 1), (5, 3, 7), (100, 64, 33), (2000, 100, 1001), (300, 257, 64), (70, 1024, 40), (1 << 17, 8, 4097)]


@pytest.mark.parametrize("rows,width,n", SHAPES)
@pytest.mark.parametrize("table_t,out_t", [(F32, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("extra,offset", [(0, 0), (1, 0), (8, 1)])
def test_embed_bits(ctx, rows, width, n, table_t, out_t, extra, offset):
    g = gen(rows + width + n)
    table = torch.randn(rows, width, generator=g).to(table_t)
    ids = torch.randint(0, rows, (n,), generator=g, dtype=torch.int32)
    ids[::7] = -1
    scale = width ** 0.5
    want = (table[ids.long().clamp(min=0)].float() * scale)
    want[ids < 0] = 0.0
    want = want.to(out_t)
    got = ctx.embed(padded(table, extra, offset), ids.to(DEV), scale=scale, padding_id=-1, out_dtype=out_t)
    assert torch.equal(got.cpu(), want)
    out = padded(torch.zeros(n, width, dtype=out_t), extra, offset)
    ctx.embed(table.to(DEV), ids.to(DEV), scale=scale, padding_id=-1, out=out)
    assert torch.equal(out.cpu(), want)
    assert ctx.stats() is not None


def test_embed_empty_nan_rows_and_row_padding(ctx):
    table = torch.randn(9, 16, device=DEV)
    table[3] = float("nan")
    table[4] = float("inf")
    assert ctx.embed(table, torch.zeros(0, dtype=torch.int32, device=DEV)).shape == (0, 16)
    ids = torch.tensor([[3, 0], [4, 8]], dtype=torch.int32, device=DEV)
    got = ctx.embed(table, ids, scale=2.0, padding_id=3)   # the padding row's content is never read
    assert got.shape == (2, 2, 16)
    assert torch.equal(got[0, 0], torch.zeros(16, device=DEV)) and torch.isinf(got[1, 0]).all()
    assert torch.equal(got[0, 1], 2.0 * table[0]) and torch.equal(got[1, 1], 2.0 * table[8])


def test_ids_outside_the_table_are_reported(pkg, ctx):
    table = torch.randn(10, 8, device=DEV)
    for bad in (10, -1, 2**31 - 1, -(1 << 31)):
        ids = torch.tensor([1, bad, 2], dtype=torch.int32, device=DEV)
        got = ctx.embed(table, ids)
        with pytest.raises(pkg.LpError) as ei:
            ctx.stats()
        assert ei.value.status == -1
        assert torch.equal(got[0], table[1]) and torch.equal(got[2], table[2]) and (got[1] == 0).all()
        grad = ctx.embed_grad(torch.ones(3, 8, device=DEV), ids, 10)
        with pytest.raises(pkg.LpError):
            ctx.stats()
        assert grad.sum().item() == 16.0
        ctx.stats()  # reported once


def test_embed_offsets_beyond_32_bits(ctx):
    rows, width = (1 << 26) + 3, 66   # 4.4e9 elements, 8.9 GB
    table = torch.zeros(rows, width, dtype=BF16, device=DEV)
    table[rows - 1] = 3.0
    table[rows - 2, 65] = 5.0
    ids = torch.tensor([rows - 1, 0, rows - 2], dtype=torch.int32, device=DEV)
    got = ctx.embed(table, ids, scale=0.5).float()
    assert (got[0] == 1.5).all() and (got[1] == 0).all() and got[2, 65] == 2.5 and got[2, :65].sum() == 0
    grad = table
    ctx.embed_grad(torch.ones(3, width, dtype=BF16, device=DEV), ids, rows, scale=2.0, grad=grad)
    assert (grad[rows - 1] == 2.0).all() and (grad[rows - 2] == 2.0).all() and (grad[0] == 2.0).all()
    assert grad[1].abs().sum() == 0 and grad[rows - 3].abs().sum() == 0
    del table, grad
    torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------ gradient
def make_ids(kind, rows, n, g):
    if kind == "uniform":
        return torch.randint(0, rows, (n,), generator=g, dtype=torch.int32)
    if kind == "one":
        return torch.full((n,), rows - 1, dtype=torch.int32)
    if kind == "hub":       # half of the ids name one row
        ids = torch.randint(0, rows, (n,), generator=g, dtype=torch.int32)
        ids[torch.rand(n, generator=g) < 0.5] = rows // 2
        return ids
    if kind == "clustered":  # all ids in a narrow range, sorted
        return (rows // 3 + torch.arange(n, dtype=torch.int32) % max(1, min(50, rows - rows // 3))).sort().values.to(torch.int32)
    ids = torch.randint(0, rows, (n,), generator=g, dtype=torch.int32)  # "padded"
    ids[torch.rand(n, generator=g) < 0.4] = -1
    return ids


def exact_grad(dout, ids, rows, scale):
    ref = torch.zeros(rows, dout.shape[1], dtype=F64)
    mag = torch.zeros(rows, dout.shape[1], dtype=F64)
    cnt = torch.zeros(rows, 1, dtype=F64)
    ok = (ids >= 0) & (ids < rows)
    i = ids[ok].long()
    d = dout[ok].double() * scale
    ref.index_add_(0, i, d)
    mag.index_add_(0, i, d.abs())
    cnt.index_add_(0, i, torch.ones(len(i), 1, dtype=F64))
    return ref, mag, cnt


@pytest.mark.parametrize("kind", ["uniform", "one", "hub", "clustered", "padded"])
@pytest.mark.parametrize("rows,width,n", [(1, 1, 1), (3, 5, 2), (50, 64, 31), (50, 64, 33), (1000, 100, 1000), (400, 37, 5000), (90000, 16, 4097), (2000, 300, 40000),
                                          (70000, 128, 70001)])
@pytest.mark.parametrize("dout_t,grad_t", [(F32, F32), (BF16, F32), (BF16, BF16)])
def test_embed_grad(ctx, kind, rows, width, n, dout_t, grad_t):
    g = gen(rows * 7 + width + n)
    ids = make_ids(kind, rows, n, g)
    dout = torch.randn(n, width, generator=g).to(dout_t)
    scale = 1.7
    ref, mag, cnt = exact_grad(dout, ids, rows, scale)
    bound = (cnt + 2) * 2.0**-24 * mag + (ref.abs() * 2.0**-8 if grad_t == BF16 else 0.0)
    dd, di = dout.to(DEV), ids.to(DEV)
    got = ctx.embed_grad(dd, di, rows, scale=scale, padding_id=-1, grad_dtype=grad_t)
    assert ((got.cpu().double() - ref).abs() <= bound).all()
    again = ctx.embed_grad(dd, di, rows, scale=scale, padding_id=-1, grad_dtype=grad_t)
    assert torch.equal(got, again)
    # accumulating into what is there
    old = torch.randn(rows, width, generator=g).to(grad_t)
    acc = old.to(DEV)
    ctx.embed_grad(dd, di, rows, scale=scale, padding_id=-1, grad=acc, accumulate=True)
    want = old.double() + ref
    bound = (cnt + 3) * 2.0**-24 * (mag + old.double().abs()) + (want.abs() * 2.0**-8 if grad_t == BF16 else 0.0)
    got = acc.cpu()
    assert ((got.double() - want).abs() <= bound).all()
    untouched = cnt[:, 0] == 0
    assert torch.equal(got[untouched], old[untouched])
    ctx.stats()


@pytest.mark.parametrize("extra,offset", [(1, 0), (8, 0), (4, 1), (2, 2)])
@pytest.mark.parametrize("dout_t,grad_t", [(F32, F32), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("n", [700, 20000])
def test_embed_grad_strided(ctx, extra, offset, dout_t, grad_t, n):
    rows, width = 500, 72
    g = gen(11)
    ids = make_ids("hub", rows, n, g)
    dout = torch.randn(n, width, generator=g).to(dout_t)
    plain = ctx.embed_grad(dout.to(DEV), ids.to(DEV), rows, scale=0.3, grad_dtype=grad_t)
    out = padded(torch.full((rows, width), 9.0, dtype=grad_t), extra, offset)
    ctx.embed_grad(padded(dout, extra, offset), ids.to(DEV), rows, scale=0.3, grad=out)
    assert torch.equal(out, plain)  # the order of the additions does not depend on the layout
    gap = torch.as_strided(out, (rows, extra), out.stride(), out.storage_offset() + width)
    assert torch.isnan(gap).all()   # nothing is written between the rows


def test_embed_grad_empty_and_nan(ctx):
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    grad = torch.full((40, 12), 7.0, device=DEV)
    ctx.embed_grad(torch.zeros(0, 12, device=DEV), none, 40, grad=grad, accumulate=True)
    assert (grad == 7.0).all()
    ctx.embed_grad(torch.zeros(0, 12, device=DEV), none, 40, grad=grad)
    assert (grad == 0.0).all()
    dout = torch.ones(3, 12, device=DEV)
    dout[1] = float("nan")   # a padded row's gradient is not read into anything
    ids = torch.tensor([4, -1, 4], dtype=torch.int32, device=DEV)
    got = ctx.embed_grad(dout, ids, 40, padding_id=-1)
    assert (got[4] == 2.0).all() and got.isfinite().all() and got.sum() == 24.0


def test_embed_grad_is_the_derivative(ctx):
    """Central differences of L = <w, embed(table)> agree with the gradient for dout = w (L is linear: exact up to rounding)."""
    g = gen(5)
    table = torch.randn(30, 24, generator=g).to(DEV)
    ids = torch.randint(0, 30, (200,), generator=g, dtype=torch.int32).to(DEV)
    w = torch.randn(200, 24, generator=g).to(DEV)
    grad = ctx.embed_grad(w, ids, 30, scale=1.5)
    for v, c in ((0, 0), (7, 23), (29, 11)):
        vals = []
        for h in (1.0, -1.0):
            t = table.clone()
            t[v, c] += h
            vals.append((w.double() * ctx.embed(t, ids, scale=1.5).double()).sum().item())
        assert abs((vals[0] - vals[1]) / 2 - grad[v, c].item()) <= 1e-5 * (1 + w.abs().sum().item() / 100)


# ------------------------------------------------------------------------------------------ orthogonalisation
def exact_orthogonalize(U, steps=5, coeffs=COEFFS, eps=1e-7):
    """From the singular values: U = P S Q^T becomes P f(f(...f(S / |S|))) Q^T."""
    P, S, Qt = torch.linalg.svd(U.double(), full_matrices=False)
    s = S / (S.square().sum(-1, keepdim=True).sqrt() + eps)
    a, b, c = coeffs
    for _ in range(steps):
        s = a * s + b * s**3 + c * s**5
    return (P * s[..., None, :]) @ Qt


def rel(a, b):
    return ((a.cpu().double() - b).norm() / b.norm()).item()


ORTH_TOL = {F32: 2e-5, BF16: 1e-2}


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 1), (2, 1, 300), (2, 300, 1), (3, 7, 5), (1, 64, 64), (5, 65, 63), (2, 128, 256), (2, 256, 128), (3, 129, 200),
                                             (1, 256, 256), (1, 417, 1000), (1, 1000, 417), (1, 640, 512), (1, 1025, 1090), (40, 30, 90)])
def test_orthogonalize(ctx, dtype, batch, rows, cols):
    U = (1e-3 * torch.randn(batch, rows, cols, generator=gen(rows * 3 + cols))).to(dtype)
    want = exact_orthogonalize(U)
    got = ctx.orthogonalize(U.to(DEV))
    for b in range(batch):
        assert rel(got[b], want[b]) <= ORTH_TOL[dtype]
    assert torch.equal(got, ctx.orthogonalize(U.to(DEV)))  # the same bits again
    ctx.stats()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["rank1", "rank3", "decay", "zero_rows", "spike", "large", "tiny"])
def test_orthogonalize_spectra(ctx, dtype, kind):
    g = gen(3)
    rows, cols = 192, 320
    U = torch.randn(rows, cols, generator=g)
    if kind in ("rank1", "rank3"):
        r = int(kind[-1])
        U = torch.randn(rows, r, generator=g) @ torch.randn(r, cols, generator=g)
    elif kind == "decay":
        P, S, Q = torch.linalg.svd(U, full_matrices=False)
        U = (P * torch.logspace(0, -4, rows)) @ Q
    elif kind == "zero_rows":
        U[::2] = 0
        U[:, 5:9] = 0
    elif kind == "spike":
        U = torch.zeros(rows, cols)
        U[17, 33] = 5.0
    elif kind == "large":
        U *= 1e30
    elif kind == "tiny":
        U *= 1e-30
    eps = 0.0 if kind == "tiny" else 1e-7
    U = U.to(dtype)
    want = exact_orthogonalize(U, eps=eps)
    got = ctx.orthogonalize(U.to(DEV), eps=eps)
    # low rank: the rounding of U itself to its own type is part of U, so nothing but the iteration's errors counts
    assert rel(got, want) <= ORTH_TOL[dtype]
    if kind == "zero_rows":
        assert (got[::2] == 0).all() and (got[:, 5:9] == 0).all()


@pytest.mark.parametrize("steps", [1, 2, 3, 8])
def test_orthogonalize_steps_and_coefficients(ctx, steps):
    U = torch.randn(100, 70, generator=gen(steps))
    for coeffs in (COEFFS, (1.875, -1.25, 0.375), (1.5, -0.5, 0.0)):
        got = ctx.orthogonalize(U.to(DEV), steps=steps, coeffs=coeffs)
        assert rel(got, exact_orthogonalize(U, steps, coeffs)) <= ORTH_TOL[F32]


def test_orthogonalize_zero_nan_inplace_strides_empty(ctx):
    assert (ctx.orthogonalize(torch.zeros(2, 70, 130, device=DEV)) == 0).all()
    U = torch.randn(4, 90, 50, generator=gen(1)).to(DEV)
    want = ctx.orthogonalize(U)
    bad = U.clone()
    bad[2, 3, 4] = float("nan")
    got = ctx.orthogonalize(bad)
    assert torch.isnan(got[2]).all()
    for b in (0, 1, 3):   # the other matrices of the batch are untouched by it
        assert torch.equal(got[b], want[b])
    big = torch.full((4, 93, 57), 2.0, device=DEV)
    view = big[:, 1:91, 3:53]
    view.copy_(U)
    ctx.orthogonalize(view, out=view)
    assert torch.equal(view, want)
    big[:, 1:91, 3:53] = 2.0
    assert (big == 2.0).all()
    shared = U[:1].expand(3, 90, 50)
    got = ctx.orthogonalize(shared)
    for b in range(3):
        assert torch.equal(got[b], want[0])
    assert ctx.orthogonalize(torch.zeros(0, 5, 6, device=DEV)).shape == (0, 5, 6)
    assert ctx.orthogonalize(torch.zeros(2, 0, 6, device=DEV)).shape == (2, 0, 6)
    many = torch.randn(2, 3, 20, 30, generator=gen(2)).to(DEV)
    assert torch.equal(ctx.orthogonalize(many)[1, 2], ctx.orthogonalize(many[1, 2]))


# ------------------------------------------------------------------------------------------ update
def layout(shapes, gap):
    mats, at = [], 0
    for r, c in shapes:
        mats.append((at, r, c))
        at += r * c + gap
    return mats, at


def exact_muon(p, m, v, g, mats, t, lr=0.02, mu=0.95, nesterov=True, weight_decay=0.01, grad_scale=0.5, adam_lr=1e-3, b1=0.9, b2=0.999, eps=1e-8):
    p, m, v, g = (x.double().clone() for x in (p, m, v, g))
    g *= grad_scale
    nm, nv = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    new = p - adam_lr * (nm / (1 - b1**t)) / ((nv / (1 - b2**t)).sqrt() + eps)
    for at, r, c in mats:
        s = slice(at, at + r * c)
        nm[s] = mu * m[s] + g[s]
        nv[s] = v[s]
        U = (g[s] + mu * nm[s]) if nesterov else nm[s]
        new[s] = (1 - lr * weight_decay) * p[s] - lr * max(1.0, c / r) ** 0.5 * exact_orthogonalize(U.view(r, c)).reshape(-1)
    return new, nm, nv


@pytest.mark.parametrize("shapes,gap", [([(64, 64)], 0), ([(128, 256), (128, 256), (256, 256), (256, 256)], 256), ([(33, 70), (70, 33), (1, 9), (9, 1)], 7),
                                        ([(40, 40 + i) for i in range(30)], 3), ([], 50)])
@pytest.mark.parametrize("nesterov", [True, False])
def test_muon_step(ctx, shapes, gap, nesterov):
    mats, n = layout(shapes, gap)
    n += 50 * (not shapes)
    g = gen(n)
    p, m, gr = 0.05 * torch.randn(n, generator=g), 1e-3 * torch.randn(n, generator=g), 1e-3 * torch.randn(n, generator=g)
    v = 1e-6 * torch.rand(n, generator=g)
    want = exact_muon(p, m, v, gr, mats, 3, nesterov=nesterov)
    d = [x.to(DEV) for x in (p, m, v, gr)]
    keep = [x.clone() for x in d]
    out = tuple(torch.full((n,), 5.0, device=DEV) for _ in range(3))
    kw = dict(t=3, matrices=mats[::-1], nesterov=nesterov, weight_decay=0.01, grad_scale=0.5)
    ctx.muon_step(*d, out=out, **kw)
    for x, y in zip(d, keep):
        assert torch.equal(x, y)
    for x, y in zip(out, want):
        assert rel(x, y) <= 1e-6
    ctx.muon_step(*d, **kw)   # in place: the same bits
    for x, y in zip(d[:3], out):
        assert torch.equal(x, y)
    if not gap:
        ctx.muon_step(d[0], d[1], None, d[3], **kw)  # the matrices cover the vector: no second moment needed


def test_muon_step_on_the_model(pkg):
    """The matrices of lp_set_model's layout, and an lp_score after the update sees the new weights."""
    import workloads as wl
    g = wl.erdos_renyi(300, 2000, seed=0)
    for arch, pred in (("sage", 0), ("gcn", 64)):
        dims = [64, 128, 64]
        ctx = pkg.Context(0)
        ctx.load_graph(g.n, g.rowptr, g.col, None, wl.node_features(g.n, 64, 0))
        n = ctx.set_model(arch, dims, max_batch=64, pred_hidden=pred)
        mats, at = [], 0
        for fi, fo in zip(dims[:-1], dims[1:]):
            for _ in range(2 if arch == "sage" else 1):
                mats.append((at, fi, fo))
                at += fi * fo
            at += fo
        if pred:
            for fi in (dims[-1], pred):
                mats.append((at, fi, pred))
                at += fi * pred + pred
            at += pred + 1
        assert at == n
        p = torch.from_numpy(wl.glorot_params(arch, dims, 0, bias_scale=0.05, pred_hidden=pred)).to(DEV)
        u, w = (torch.from_numpy(x[:64].copy()).to(DEV) for x in wl.undirected_edge_list(g))
        grads, loss = torch.zeros(n, device=DEV), torch.zeros(1, device=DEV)
        _, nd = ctx.sample_negatives(seed=1, step=0, k=1, pos_src=u)
        ctx.train_step(p, u, w, None, nd, 1, loss, grads)
        before = ctx.score(p, u, w)
        m, v = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
        explicit = tuple(torch.empty_like(p) for _ in range(3))
        ctx.muon_step(p, m, v, grads, t=1, matrices=mats, out=explicit)
        ctx.muon_step(p, m, v, grads, t=1)
        assert torch.equal(p, explicit[0]) and torch.equal(m, explicit[1]) and torch.equal(v, explicit[2])
        after = ctx.score(p, u, w)
        assert not torch.equal(before, after)
        ctx.invalidate_embeddings()
        assert torch.equal(after, ctx.score(p, u, w))
        ctx.close()


# ------------------------------------------------------------------------------------------ streams, workspace, refusals
def test_other_streams(pkg):
    """Called from another current stream than the context's, the operators wait for what that stream has enqueued."""
    side = torch.cuda.Stream()
    ctx = pkg.Context(0, stream=side)
    ids = torch.randint(0, 5000, (20000,), dtype=torch.int32, device=DEV)
    for rep in range(3):
        big = torch.randn(4000, 4000, device=DEV)
        for _ in range(4):
            big = big @ big * 1e-2
        dout = torch.ones(20000, 64, device=DEV) * (rep + 1)
        got = ctx.embed_grad(dout, ids, 5000)
        del dout
        assert got.double().sum().item() == 20000 * 64 * (rep + 1)
        U = torch.randn(64, 96, device=DEV)
        O = ctx.orthogonalize(U)
        assert rel(O, exact_orthogonalize(U.cpu())) <= 2e-5
    ctx.close()


def test_workspace_is_kept_and_counted(pkg):
    c = pkg.Context(0)
    base = c.stats().workspace_bytes
    U = torch.randn(512, 512, device=DEV)
    c.orthogonalize(U)
    first = c.stats().workspace_bytes
    assert first > base
    c.orthogonalize(U)
    c.orthogonalize(U[:100, :100])
    assert c.stats().workspace_bytes == first
    c.close()


def test_refusals(pkg, ctx):
    table, ids = torch.zeros(10, 8, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
    U = torch.zeros(6, 8, device=DEV)
    vec = torch.zeros(48, device=DEV)
    calls = [
        lambda: ctx.embed(table, ids.long()),
        lambda: ctx.embed(table.double(), ids),
        lambda: ctx.embed(table.half(), ids),
        lambda: ctx.embed(table.cpu(), ids),
        lambda: ctx.embed(table, ids.cpu()),
        lambda: ctx.embed(table.t(), ids),
        lambda: ctx.embed(table[0], ids),
        lambda: ctx.embed(table[:1].expand(10, 8), ids),
        lambda: ctx.embed(table.bfloat16(), ids, out_dtype=F32),
        lambda: ctx.embed(table, ids, scale=float("nan")),
        lambda: ctx.embed(table, ids, out=torch.zeros(3, 8, device=DEV)),
        lambda: ctx.embed(table, ids[::2]),
        lambda: ctx.embed_grad(torch.zeros(3, 8, device=DEV), ids, 10),
        lambda: ctx.embed_grad(torch.zeros(4, 8, device=DEV), ids, 0),
        lambda: ctx.embed_grad(torch.zeros(4, 8, device=DEV), ids, 10, grad_dtype=BF16),
        lambda: ctx.embed_grad(torch.zeros(4, 8, device=DEV), ids, 10, accumulate=True),
        lambda: ctx.embed_grad(torch.zeros(1, 8, device=DEV).expand(4, 8), ids, 10),
        lambda: ctx.orthogonalize(U.double()),
        lambda: ctx.orthogonalize(U[0]),
        lambda: ctx.orthogonalize(U.t()),
        lambda: ctx.orthogonalize(U, steps=0),
        lambda: ctx.orthogonalize(U, steps=65),
        lambda: ctx.orthogonalize(U, eps=-1.0),
        lambda: ctx.orthogonalize(U, eps=float("nan")),
        lambda: ctx.orthogonalize(U, coeffs=(5.0, 0.0, 0.0)),
        lambda: ctx.orthogonalize(U, coeffs=(float("inf"), 0.0, 0.0)),
        lambda: ctx.orthogonalize(U, out=torch.zeros(8, 6, device=DEV)),
        lambda: ctx.orthogonalize(U, out=torch.zeros(6, 8, dtype=BF16, device=DEV)),
        lambda: ctx.muon_step(vec, vec, vec, vec, t=1, matrices=[(1, 6, 8)]),
        lambda: ctx.muon_step(vec, vec, vec, vec, t=1, matrices=[(0, 6, 4), (20, 2, 2)]),
        lambda: ctx.muon_step(vec, vec, vec, vec, t=1, matrices=[(-1, 2, 2)]),
        lambda: ctx.muon_step(vec, vec, vec, vec, t=1, matrices=[(0, 0, 8)]),
        lambda: ctx.muon_step(vec, vec, None, vec, t=1, matrices=[(0, 6, 4)]),
        lambda: ctx.muon_step(vec, vec, vec, vec, t=0, matrices=[(0, 6, 4)]),
        lambda: ctx.muon_step(vec, vec, vec, vec, t=1, matrices=[(0, 6, 8)], lr=float("nan")),
        lambda: ctx.muon_step(vec, vec[:40], vec, vec, t=1, matrices=[(0, 6, 4)]),
        lambda: ctx.muon_step(vec, vec, vec, vec, t=1),  # no model
    ]
    for i, call in enumerate(calls):
        with pytest.raises(pkg.LpError):
            call()
            pytest.fail(f"call {i} was not refused")
    ctx.stats()
    assert (vec == 0).all() and (table == 0).all()
    lib = pkg.load_library()
    assert lib.lp_embed(None, 0, None, 1, 1, 1, None, 0, 0, 1.0, 0, None, 1) == -1
    assert lib.lp_embed(ctx.h, 0, table.data_ptr() + 2, 10, 8, 8, ids.data_ptr(), 4, -1, 1.0, 0, table.data_ptr(), 8) == -1
    assert lib.lp_orthogonalize(ctx.h, 0, 2, 6, 8, U.data_ptr(), 8, 48, 5, None, 1e-7, U.data_ptr(), 8, 40) == -1


def test_bounded_wait_of_the_products(pkg):
    """A product that waits for bytes that never come gives up, is reported once, and the context stays usable."""
    c = pkg.Context(0)
    U = torch.randn(64, 64, device=DEV)
    want = c.orthogonalize(U)
    c.set_wait_limit(2_000_000, 16)
    c.orthogonalize(U)
    with pytest.raises(pkg.LpError) as ei:
        c.stats()
    assert ei.value.status == -6
    c.set_wait_limit(2_000_000_000, 0)
    c.stats()
    assert torch.equal(c.orthogonalize(U), want)
    c.close()


# ------------------------------------------------------------------------------------------ matrices of up to 128 x 128, one block each
def fp32_orthogonalize(U):
    """The iteration in FP32 matrix products."""
    X = U if U.shape[0] <= U.shape[1] else U.T
    X = X / (X.norm() + 1e-7)
    a, b, c = COEFFS
    for _ in range(5):
        A = X @ X.T
        X = a * X + (b * A + c * (A @ A)) @ X
    return X if U.shape[0] <= U.shape[1] else X.T


@pytest.mark.parametrize("kind", ["rank1", "rank3", "decay", "zero_rows", "spike", "large", "tiny"])
@pytest.mark.parametrize("rows,cols", [(64, 64), (37, 128), (128, 128), (128, 50)])
def test_small_orthogonalize_spectra(ctx, rows, cols, kind):
    """No further from 64 bits than FP32 matrix products are where those miss the tolerance (directions that U lacks)."""
    g = gen(rows + cols)
    U = torch.randn(rows, cols, generator=g)
    if kind in ("rank1", "rank3"):
        r = int(kind[-1])
        U = torch.randn(rows, r, generator=g) @ torch.randn(r, cols, generator=g)
    elif kind == "decay":
        P, S, Q = torch.linalg.svd(U, full_matrices=False)
        U = (P * torch.logspace(0, -4, S.numel())) @ Q
    elif kind == "zero_rows":
        U[::2] = 0
    elif kind == "spike":
        U = torch.zeros(rows, cols)
        U[17, 33] = 5.0
    elif kind in ("large", "tiny"):
        U *= 1e30 if kind == "large" else 1e-30
    eps = 0.0 if kind == "tiny" else 1e-7
    want = exact_orthogonalize(U, eps=eps)
    tol = ORTH_TOL[F32]
    if kind not in ("large", "tiny"):  # whose squares leave FP32
        tol = max(tol, rel(fp32_orthogonalize(U), want))
    assert rel(ctx.orthogonalize(U.to(DEV), eps=eps), want) <= tol
    assert rel(ctx.orthogonalize(U.to(DEV).to(BF16), eps=eps), exact_orthogonalize(U.to(BF16), eps=eps)) <= ORTH_TOL[BF16]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(5, 9), (9, 5), (1, 128), (128, 1), (64, 65), (100, 128), (128, 127)])
def test_small_orthogonalize_many_strided(ctx, rows, cols, dtype):
    """More matrices than SMs, rows apart, results into another layout: each the bits of the matrix alone."""
    n = 300
    U = torch.randn(n, rows, cols, generator=gen(rows * cols)).to(dtype).to(DEV)
    want = ctx.orthogonalize(U)
    assert (torch.stack([torch.as_tensor(rel(want[i], exact_orthogonalize(U[i].cpu()))) for i in range(0, n, 37)]) <= ORTH_TOL[dtype]).all()
    assert torch.equal(ctx.orthogonalize(U[211]), want[211])
    wide = torch.zeros(n, rows + 1, cols + 3, dtype=dtype, device=DEV)
    wide[:, :rows, 1 : cols + 1] = U
    out = torch.full((n, rows + 2, cols + 5), 7.0, dtype=dtype, device=DEV)
    ctx.orthogonalize(wide[:, :rows, 1 : cols + 1], out=out[:, 1 : rows + 1, 2 : cols + 2])
    assert torch.equal(out[:, 1 : rows + 1, 2 : cols + 2], want)
    out[:, 1 : rows + 1, 2 : cols + 2] = 7.0
    assert (out == 7.0).all()


@pytest.mark.parametrize("shapes", [[(64, 128), (128, 64), (128, 128)], [(1, 1), (127, 3), (3, 127), (64, 64)], [(128, 129), (64, 64)]])
def test_small_muon_step(ctx, shapes):
    """All matrices small, and one that is not beside one that is; the stretches between them take Adam steps."""
    mats, n = layout(shapes, 1500)
    g = gen(n)
    p, m, gr = 0.05 * torch.randn(n, generator=g), 1e-3 * torch.randn(n, generator=g), 1e-3 * torch.randn(n, generator=g)
    v = 1e-6 * torch.rand(n, generator=g)
    want = exact_muon(p, m, v, gr, mats, 4)
    d = [x.to(DEV) for x in (p, m, v, gr)]
    out = tuple(torch.full((n,), 5.0, device=DEV) for _ in range(3))
    kw = dict(t=4, matrices=mats, weight_decay=0.01, grad_scale=0.5)
    ctx.muon_step(*d, out=out, **kw)
    for x, y in zip(out, want):
        assert rel(x, y) <= 1e-6
    ctx.muon_step(*d, **kw)
    for x, y in zip(d[:3], out):
        assert torch.equal(x, y)


def test_bounded_wait_of_the_chained_products(pkg):
    c = pkg.Context(0)
    U = torch.randn(160, 160, device=DEV)
    want = c.orthogonalize(U)
    c.set_wait_limit(2_000_000, 16)
    c.orthogonalize(U)
    with pytest.raises(pkg.LpError) as ei:
        c.stats()
    assert ei.value.status == -6
    c.set_wait_limit(2_000_000_000, 0)
    assert torch.equal(c.orthogonalize(U), want)
    c.close()


@pytest.mark.parametrize("rows,width,n,dtype", [(300_000, 64, 40, F32), (1_200_000, 33, 700, BF16), (600_000, 37, 20_000, F32), (1_100_001, 31, 30_001, BF16)])
def test_embed_grad_of_a_large_sparse_table(ctx, rows, width, n, dtype):
    """Large gradients that few ids name: the bits of the same call with rows apart, which clears row by row; nothing stale stays."""
    g = gen(n)
    ids = torch.randint(0, rows, (n,), generator=g, dtype=torch.int32)
    ids[: n // 3] = ids[0]
    ids[-1] = rows - 1
    dout = torch.randn(n, width, generator=g).to(dtype).to(DEV)
    ids = ids.to(DEV)
    grad = torch.full((rows, width), float("nan"), dtype=dtype, device=DEV)
    ctx.embed_grad(dout, ids, rows, scale=2.0, grad=grad)
    apart = torch.full((rows, width + 1), float("nan"), dtype=dtype, device=DEV)
    ctx.embed_grad(dout, ids, rows, scale=2.0, grad=apart[:, :width])
    assert torch.equal(grad, apart[:, :width])
    named = torch.zeros(rows, dtype=torch.bool, device=DEV)
    named[ids.long()] = True
    assert (grad[~named] == 0).all()
    want = torch.zeros(rows, width, dtype=torch.float64, device=DEV).index_add_(0, ids.long(), 2.0 * dout.double())[named]
    size = torch.zeros(rows, width, dtype=torch.float64, device=DEV).index_add_(0, ids.long(), 2.0 * dout.double().abs())[named]
    # FP32 sums of k terms: k 2^-24 of the sum of magnitudes, and one rounding to BF16
    assert ((grad[named].double() - want).abs() <= n * 2.0**-24 * size + (2.0**-8 * want.abs() if dtype == BF16 else 0.0)).all()


@pytest.mark.parametrize("rows,width,n,dtype", [(300, 33, 20_000, F32), (2000, 450, 9_001, BF16), (1, 700, 8_500, F32), (2200, 64, 8_800, BF16)])
def test_embed_grad_of_a_small_dense_table(ctx, rows, width, n, dtype):
    """Many more ids than rows, which clears everything first: stale rows go, what lies between the rows stays."""
    g = gen(rows + n)
    ids = torch.randint(0, max(1, rows - 7), (n,), generator=g, dtype=torch.int32).to(DEV)  # the last rows have no ids
    dout = torch.randn(n, width, generator=g).to(dtype).to(DEV)
    grad = torch.full((rows, width), float("nan"), dtype=dtype, device=DEV)
    ctx.embed_grad(dout, ids, rows, scale=0.5, grad=grad)
    apart = torch.full((rows, width + 5), 3.0, dtype=dtype, device=DEV)
    ctx.embed_grad(dout, ids, rows, scale=0.5, grad=apart[:, 2 : width + 2])
    assert torch.equal(apart[:, 2 : width + 2], grad)
    assert (apart[:, :2] == 3.0).all() and (apart[:, width + 2 :] == 3.0).all()
    want = torch.zeros(rows, width, dtype=torch.float64, device=DEV).index_add_(0, ids.long(), 0.5 * dout.double())
    size = torch.zeros(rows, width, dtype=torch.float64, device=DEV).index_add_(0, ids.long(), 0.5 * dout.double().abs())
    assert ((grad.double() - want).abs() <= n * 2.0**-24 * size + (2.0**-8 * want.abs() if dtype == BF16 else 0.0)).all()
