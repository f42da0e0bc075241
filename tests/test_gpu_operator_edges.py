"""Edges of the embedding and orthogonalisation operators: waits that run out, replayed graphs, zeros, layouts, error reports, and
the kernel of the large products.

Tolerances are those of test_gpu_operators.py unless a test derives its own.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F64 = torch.float32, torch.bfloat16, torch.float64
COEFFS = (3.4445, -4.7750, 2.0315)
ORTH_TOL = {F32: 2e-5, BF16: 1e-2}


@pytest.fixture(scope="module")
def pkg():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__ as ge
    ge.build()
    import paper_2506_20818_b200 as p
    return p


@pytest.fixture
def ctx(pkg):
    c = pkg.Context(0)
    yield c
    c.close()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rel(a, b):
    return ((a.cpu().double() - b).norm() / b.norm()).item()


# ------------------------------------------------------------------------------------------ waits that run out
@pytest.mark.parametrize("n", [20_000, 300_000])
def test_sort_that_gives_up_is_reported_and_reads_nothing_outside(pkg, ctx, n):
    """The first tile of ids publishes nothing, so every other tile's wait runs out: reported once as LP_ETIMEOUT, and the context
    stays usable.  Positions that no tile wrote hold the products of another operator here (any 32 bits), which must not be
    followed into dout."""
    rows, width = 5000, 40
    ids = torch.randint(0, rows, (n,), generator=gen(n), dtype=torch.int32).to(DEV)
    dout = torch.ones(n, width, device=DEV)
    want = torch.bincount(ids, minlength=rows).float()[:, None].expand(rows, width)
    assert torch.equal(ctx.embed_grad(dout, ids, rows), want)   # counts below 2^24: exact
    ctx.orthogonalize(torch.randn(1024, 1200, generator=gen(0)).to(DEV))   # fills the workspace with numbers that are no positions
    ctx.set_wait_limit(2_000_000, 16)
    got = ctx.embed_grad(dout, ids, rows)
    with pytest.raises(pkg.LpError) as ei:
        ctx.stats()
    assert ei.value.status == -6
    assert got.shape == (rows, width)
    ctx.stats()                              # reported once
    ctx.set_wait_limit(2_000_000_000, 0)
    assert torch.equal(ctx.embed_grad(dout, ids, rows), want)
    ctx.stats()


# ------------------------------------------------------------------------------------------ captured graphs
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(64, 64), (160, 192), (512, 300)])
def test_orthogonalize_in_a_replayed_graph(pkg, rows, cols, dtype):
    """A captured call gives the bits of an eager one in every replay, and leaves an eager call after it right: (64, 64) is taken by the
    one-block kernel, the others by the chain kernel, whose blocks wait for counters in global memory."""
    side = torch.cuda.Stream()
    c = pkg.Context(0, stream=side)
    g = gen(rows)
    U = torch.zeros(rows, cols, dtype=dtype, device=DEV)
    O = torch.zeros_like(U)
    inputs = [torch.randn(rows, cols, generator=g).to(dtype).to(DEV) for _ in range(5)]
    torch.cuda.synchronize()
    want = [c.orthogonalize(x) for x in inputs]   # also the workspace
    torch.cuda.synchronize()
    launches = c.stats().kernel_launches
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.orthogonalize(U, out=O)
    assert c.stats().kernel_launches == launches + 1
    for x, w in zip(inputs, want):
        with torch.cuda.stream(side):
            U.copy_(x)
            O.fill_(float("nan"))
            graph.replay()
            graph.replay()
        side.synchronize()
        assert torch.equal(O, w)
        assert torch.equal(c.orthogonalize(x), w)
    c.stats()
    del graph
    c.close()


def test_muon_step_in_a_replayed_graph(pkg):
    side = torch.cuda.Stream()
    c = pkg.Context(0, stream=side)
    mats = [(0, 128, 256), (128 * 256 + 256, 256, 200)]
    n = mats[1][0] + 256 * 200 + 77
    g = gen(1)
    start = [0.05 * torch.randn(n, generator=g), 1e-3 * torch.randn(n, generator=g), 1e-6 * torch.rand(n, generator=g), 1e-3 * torch.randn(n, generator=g)]
    eager = [x.to(DEV) for x in start]
    replayed = [x.to(DEV) for x in start]
    torch.cuda.synchronize()
    for _ in range(4):
        c.muon_step(*eager, t=2, matrices=mats)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.muon_step(*replayed, t=2, matrices=mats)
    with torch.cuda.stream(side):
        for _ in range(4):
            graph.replay()
    side.synchronize()
    for x, y in zip(eager, replayed):
        assert torch.equal(x, y)
    c.stats()
    del graph
    c.close()


def test_workspace_of_a_captured_call_survives_larger_calls(pkg):
    """The block that a graph was captured with stays where it is when a later call makes the workspace grow; a capture that would
    have to allocate is refused and can go on."""
    side = torch.cuda.Stream()
    c = pkg.Context(0, stream=side)
    rows, width, n = 3000, 48, 20_000
    g = gen(8)
    ids = torch.randint(0, rows, (n,), generator=g, dtype=torch.int32).to(DEV)
    dout = torch.randn(n, width, generator=g).to(DEV)
    U = torch.randn(200, 260, generator=g).to(DEV)
    grad, O = torch.zeros(rows, width, device=DEV), torch.zeros_like(U)
    big = torch.randn(1500, 1600, generator=g).to(DEV)
    torch.cuda.synchronize()
    want_grad, want_O = c.embed_grad(dout, ids, rows), c.orthogonalize(U)
    torch.cuda.synchronize()
    before = c.stats().workspace_bytes
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.embed_grad(dout, ids, rows, grad=grad)
        c.orthogonalize(U, out=O)
        with pytest.raises(pkg.LpError) as ei:
            c.orthogonalize(big, out=big)
    assert ei.value.status == -2   # LP_ESTATE
    c.orthogonalize(big, out=big)      # grows
    assert c.stats().workspace_bytes > 2 * before
    reuse = [torch.full((before,), 255, dtype=torch.uint8, device=DEV) for _ in range(3)]   # whatever was given back is written over
    with torch.cuda.stream(side):
        graph.replay()
    side.synchronize()
    assert torch.equal(grad, want_grad) and torch.equal(O, want_O)
    assert all((x == 255).all() for x in reuse)
    c.stats()
    del graph
    c.close()


# ------------------------------------------------------------------------------------------ zeros, infinities
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("batch,rows,cols", [(3, 64, 40), (3, 150, 200), (2, 2100, 2300)])   # one-block, chain and pair kernel
def test_zeros_with_eps_zero_stay_zeros(ctx, dtype, batch, rows, cols):
    U = torch.randn(batch, rows, cols, generator=gen(rows)).to(dtype).to(DEV)
    U[1] = 0
    launches = ctx.stats().kernel_launches
    got = ctx.orthogonalize(U, eps=0.0)
    assert ctx.stats().kernel_launches - launches == (1 if rows < 2000 else 2 + 3 * 5)   # which kernel it was
    assert (got[1] == 0).all()
    assert got.isfinite().all() and (got[0] != 0).any()
    U[1, 3, 5] = float("inf")   # what is not finite is not hidden
    got = ctx.orthogonalize(U, eps=0.0)
    assert got[1].isnan().all() and got[0].isfinite().all()


def test_muon_step_of_a_frozen_layer_with_eps_zero(ctx):
    mats = [(0, 48, 96), (48 * 96, 256, 160)]
    n = 48 * 96 + 256 * 160
    g = gen(2)
    p = torch.randn(n, generator=g).to(DEV)
    m, gr = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    gr[48 * 96:] = torch.randn(256 * 160, generator=g).to(DEV)   # the first matrix has no gradient and no momentum
    new = ctx.muon_step(p, m, None, gr, t=1, matrices=mats, ns_eps=0.0, lr=0.5, weight_decay=0.25, out=(torch.empty_like(p), torch.empty_like(m), None))
    assert torch.equal(new[0][:48 * 96], p[:48 * 96] * 0.875) and new[0].isfinite().all()
    assert not torch.equal(new[0][48 * 96:], p[48 * 96:] * 0.875)


# ------------------------------------------------------------------------------------------ error reports
def test_bad_embedding_ids_are_no_other_calls_error(pkg, ctx):
    """An id outside the table is reported by the next stats() and by nothing else: candidates set meanwhile are not refused for it,
    loading and sparsifying a graph do not forget it, and a step's own report does not swallow it."""
    import workloads as wl
    g = wl.erdos_renyi(200, 1500, seed=0)
    table = torch.randn(10, 8, device=DEV)
    bad = torch.tensor([1, 10, 2], dtype=torch.int32, device=DEV)

    def report():
        with pytest.raises(pkg.LpError) as ei:
            ctx.stats()
        assert ei.value.status == -1 and "table" in str(ei.value)
        ctx.stats()   # once

    ctx.embed(table, bad)
    ctx.load_graph(g.n, g.rowptr, g.col, None, wl.node_features(g.n, 16, 0))
    report()
    ctx.embed_grad(torch.ones(3, 8, device=DEV), bad, 10)
    candidates = torch.arange(50, dtype=torch.int32, device=DEV)
    ctx.set_candidates(candidates)
    report()
    ctx.embed(table, bad)
    ctx.sparsify(0.5, 1)
    report()
    ctx.embed(table, bad)
    with pytest.raises(pkg.LpError):
        ctx.set_candidates(torch.tensor([0, 200], dtype=torch.int32, device=DEV))   # a bad candidate is still one
    report()


# ------------------------------------------------------------------------------------------ layouts
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,rows,cols", [(3, 40, 64), (5, 90, 33), (3, 300, 160), (2, 2100, 2111)])
def test_orthogonalize_of_interleaved_matrices(pkg, ctx, heads, rows, cols, dtype):
    """Matrices whose rows lie between one another's ([heads, rows, cols] as a view of [rows, heads, cols]): out of place and in place."""
    x = torch.randn(rows, heads, cols + 1, generator=gen(cols)).to(dtype).to(DEV)
    view = x.transpose(0, 1)[:, :, :cols]
    want = ctx.orthogonalize(view.contiguous())
    assert torch.equal(ctx.orthogonalize(view), want)
    last = x[:, :, cols].clone()
    ctx.orthogonalize(view, out=view)
    assert torch.equal(view, want) and torch.equal(x[:, :, cols], last)
    lib = pkg.load_library()
    prec = 0 if dtype == F32 else 1
    assert pkg.LP_FP32 == 0 and pkg.LP_BF16 == 1
    bad = lambda ld, stride: lib.lp_orthogonalize(ctx.h, prec, heads, rows, cols, x.data_ptr(), heads * (cols + 1), cols + 1, 5, None, 1e-7, x.data_ptr(), ld, stride)
    assert bad(heads * (cols + 1), cols - 1) == -1 and bad(heads * (cols + 1) - 2, cols + 1) == -1 and bad(heads * (cols + 1), 0) == -1


# ------------------------------------------------------------------------------------------ arguments beyond 32 bits
def test_numbers_beyond_32_bits_are_refused_and_not_cut(pkg, ctx):
    """2^32 is not id 0, 2^32 + 5 steps are not five, a matrix of 2^32 + 4 rows is not one of four."""
    table = torch.randn(10, 8, device=DEV)
    ids = torch.zeros(4, dtype=torch.int32, device=DEV)
    U, vec = torch.randn(4, 4, device=DEV), torch.zeros(16, device=DEV)
    for call in (lambda: ctx.embed(table, ids, padding_id=1 << 32), lambda: ctx.embed(table, ids, padding_id=-(1 << 32)),
                 lambda: ctx.embed_grad(torch.ones(4, 8, device=DEV), ids, 10, padding_id=1 << 32), lambda: ctx.orthogonalize(U, steps=(1 << 32) + 5),
                 lambda: ctx.muon_step(vec, vec, vec, vec, t=1, matrices=[(0, 4, 4)], steps=(1 << 32) + 5),
                 lambda: ctx.muon_step(vec, vec, vec, vec, t=1, matrices=[(0, (1 << 32) + 4, 4)])):
        with pytest.raises(pkg.LpError) as ei:
            call()
        assert ei.value.status == -1
    assert (ctx.embed(table, ids, padding_id=0) == 0).all()
    assert torch.equal(ctx.embed(table, ids, padding_id=pkg.LP_NO_PADDING), table[:1].expand(4, 8))
    a, b = vec.clone(), vec.clone()
    g = torch.randn(16, device=DEV)
    ctx.muon_step(a, torch.zeros_like(a), None, g, t=1, matrices=[(0, 4, 4)])
    ctx.muon_step(b, torch.zeros_like(b), None, g, t=1, matrices=[pkg.Matrix(0, 4, 4)])
    assert torch.equal(a, b) and (a != 0).all()
    ctx.stats()


# ------------------------------------------------------------------------------------------ workspace of an update
def test_workspace_of_an_update_follows_its_matrices(ctx):
    """One long matrix does not make the others' arenas as wide as itself: 100 x 100,000 takes about 0.2 GB and 2048 x 2048 0.1 GB, in
    common arenas 3.5 GB.  The results are those of calls with one matrix each: the same bits for the one that shares no launch, and
    within the tolerance of an update (1e-6) on both sides where the company decides which kernel multiplies."""
    shapes = [(100, 100_000), (2048, 2048), (70, 64)]
    mats, n = [], 0
    for r, c in shapes:
        mats.append((n, r, c))
        n += r * c + 5
    g = gen(4)
    p, m, v, gr = (torch.randn(n, generator=g).to(DEV) for _ in range(4))
    v.abs_()
    base = ctx.stats().workspace_bytes
    new = ctx.muon_step(p, m, v, gr, t=3, matrices=mats, out=tuple(torch.empty_like(p) for _ in range(3)))
    assert ctx.stats().workspace_bytes - base < 400e6
    for i, (at, r, c) in enumerate(mats):
        end = at + r * c + 5   # the matrix and the five numbers behind it
        alone = ctx.muon_step(p[at:end].clone(), m[at:end].clone(), v[at:end].clone(), gr[at:end].clone(), t=3, matrices=[(0, r, c)])
        assert rel(new[0][at:end], alone[0].double().cpu()) <= (0.0 if i == 0 else 2e-6)
        assert torch.equal(new[1][at:end], alone[1]) and torch.equal(new[2][at:end], alone[2])
    ctx.stats()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_small_matrices_need_no_workspace(ctx, dtype):
    """They stay on chip, so 70,000 of them (more than one launch takes) take no device memory beside themselves."""
    U = torch.randn(70_000, 20, 33, generator=gen(3)).to(dtype).to(DEV)
    base = ctx.stats().workspace_bytes
    before = ctx.stats().kernel_launches
    got = ctx.orthogonalize(U)
    assert ctx.stats().kernel_launches - before == 2 and ctx.stats().workspace_bytes == base
    want = iterate(U)
    err = (got.double() - want).norm(dim=(-2, -1)) / want.norm(dim=(-2, -1))
    assert (err <= ORTH_TOL[dtype]).all()
    for i in (0, 65_535, 65_536, 69_999):
        assert torch.equal(ctx.orthogonalize(U[i]), got[i])
    p, m, g = (torch.randn(128 * 64 * 3, generator=gen(k)).to(DEV) for k in range(3))
    ctx.muon_step(p, m, None, g, t=1, matrices=[(i * 128 * 64, 128, 64) for i in range(3)])
    assert ctx.stats().workspace_bytes == base


def test_workspace_that_cannot_be_had_fails_that_call_alone(pkg, ctx):
    """LP_ENOMEM, nothing written, and the next call is as before."""
    U = torch.randn(100, 140, generator=gen(6)).to(DEV)
    want = ctx.orthogonalize(U)
    n = 12_000   # 3.5 GB of workspace
    p, m, g = (torch.ones(n * n, device=DEV) for _ in range(3))
    torch.cuda.empty_cache()
    free, _ = torch.cuda.mem_get_info()
    taken = torch.empty(max(0, free - (2 << 30)), dtype=torch.uint8, device=DEV)   # 2 GB are left
    try:
        with pytest.raises(pkg.LpError) as ei:
            ctx.muon_step(p, m, None, g, t=1, matrices=[(0, n, n)])
        assert ei.value.status == -3
        assert (p == 1.0).all() and (m == 1.0).all()
        assert torch.equal(ctx.orthogonalize(U), want)
        ctx.stats()
    finally:
        del taken
        torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------ the kernel of the large products
# It is the only one that launches every product by itself, so the launches of a call tell that it was reached.
def iterate(U, steps=5, eps=1e-7, dtype=F64):
    """The iteration as it is written down, in `dtype`, on the GPU."""
    tall = U.shape[-2] > U.shape[-1]
    X = (U.mT if tall else U).to(dtype)
    X = X / (torch.linalg.matrix_norm(X, keepdim=True) + eps)
    a, b, c = COEFFS
    for _ in range(steps):
        A = X @ X.mT
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.mT if tall else X


def by_products(ctx, call, steps=5, groups=1):
    before = ctx.stats().kernel_launches
    got = call()
    assert ctx.stats().kernel_launches - before == groups * (2 + 3 * steps)
    return got


def gpu_rel(a, b):
    return ((a.double() - b).norm() / b.norm()).item()


LARGE = [(F32, 1, 2049, 2111), (F32, 1, 2111, 2049), (F32, 1, 1090, 1025), (F32, 1, 1600, 1700), (F32, 6, 900, 1100), (F32, 5, 1100, 900), (F32, 16, 520, 530),
         (BF16, 1, 2049, 2111), (BF16, 1, 2111, 2049), (BF16, 1, 1600, 1700), (BF16, 6, 900, 1100), (BF16, 5, 1100, 900), (BF16, 3, 1500, 1400), (BF16, 3, 1401, 1499)]


@pytest.mark.parametrize("dtype,batch,rows,cols", LARGE)
def test_large_orthogonalize(ctx, dtype, batch, rows, cols):
    """Wide, tall, batches, odd sizes; into rows apart with even and odd pitch and base; in place."""
    U = (1e-3 * torch.randn(batch, rows, cols, generator=gen(rows + cols))).to(dtype).to(DEV)
    want = iterate(U)
    got = by_products(ctx, lambda: ctx.orthogonalize(U))
    for i in range(batch):
        assert gpu_rel(got[i], want[i]) <= ORTH_TOL[dtype]
    assert torch.equal(ctx.orthogonalize(U), got)
    for extra, first in ((2, 0), (3, 1), (8, 8), (5, 2)):
        wide = torch.full((batch, rows + 1, cols + extra + first), 7.0, dtype=dtype, device=DEV)
        out = wide[:, :rows, first:first + cols]
        ctx.orthogonalize(U, out=out)
        assert torch.equal(out, got)
        out.copy_(U)
        ctx.orthogonalize(out, out=out)
        assert torch.equal(out, got)
        out.fill_(7.0)
        assert (wide == 7.0).all()
    ctx.stats()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(1600, 1700), (1711, 1600)])
@pytest.mark.parametrize("kind", ["rank1", "rank3", "zero_rows", "spike", "large", "tiny"])
def test_large_orthogonalize_spectra(ctx, dtype, rows, cols, kind):
    """No further from 64 bits than FP32 matrix products are where those miss the tolerance (directions that U lacks)."""
    g = gen(rows)
    U = torch.randn(rows, cols, generator=g)
    if kind in ("rank1", "rank3"):
        r = int(kind[-1])
        U = torch.randn(rows, r, generator=g) @ torch.randn(r, cols, generator=g)
    elif kind == "zero_rows":
        U[::2] = 0
        U[:, 5:9] = 0
    elif kind == "spike":
        U = torch.zeros(rows, cols)
        U[17, 33] = 5.0
    elif kind in ("large", "tiny"):
        U *= 1e30 if kind == "large" else 1e-30
    eps = 0.0 if kind == "tiny" else 1e-7
    U = U.to(dtype).to(DEV)
    want = iterate(U, eps=eps)
    got = by_products(ctx, lambda: ctx.orthogonalize(U, eps=eps))
    tol = ORTH_TOL[dtype]
    if dtype == F32 and kind not in ("large", "tiny"):  # whose squares leave FP32
        tol = max(tol, gpu_rel(iterate(U, dtype=F32), want))
    assert gpu_rel(got, want) <= tol
    if kind == "zero_rows":
        assert (got[::2] == 0).all() and (got[:, 5:9] == 0).all()


@pytest.mark.parametrize("steps", [1, 2, 7])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_orthogonalize_steps(ctx, dtype, steps):
    U = torch.randn(2, 1700, 1500, generator=gen(steps)).to(dtype).to(DEV)
    got = by_products(ctx, lambda: ctx.orthogonalize(U, steps=steps), steps)
    want = iterate(U, steps)
    assert max(gpu_rel(got[i], want[i]) for i in range(2)) <= ORTH_TOL[dtype]


@pytest.mark.parametrize("shapes,gap", [([(1000, 1999), (1999, 1500), (1500, 417)], 333), ([(1600, 1600), (64, 1000), (1000, 30)], 0), ([(1801, 1799)], 5000)])
@pytest.mark.parametrize("nesterov", [True, False])
def test_large_muon_step(ctx, shapes, gap, nesterov):
    """Several matrices in one launch, wide and tall, Adam steps between them; out of place and in place."""
    mats, n = [], 0
    for r, c in shapes:
        n += gap
        mats.append((n, r, c))
        n += r * c
    n += gap
    g = gen(n)
    p, m, gr = 0.05 * torch.randn(n, generator=g), 1e-3 * torch.randn(n, generator=g), 1e-3 * torch.randn(n, generator=g)
    v = 1e-6 * torch.rand(n, generator=g)
    d = [x.to(DEV) for x in (p, m, v, gr)]
    P, M, V, G = (x.double() for x in d)
    G = 0.5 * G
    lr, mu, wd, b1, b2, t = 0.02, 0.95, 0.01, 0.9, 0.999, 3
    nm, nv = b1 * M + (1 - b1) * G, b2 * V + (1 - b2) * G * G
    new = P - 1e-3 * (nm / (1 - b1**t)) / ((nv / (1 - b2**t)).sqrt() + 1e-8)
    for at, r, c in mats:
        s = slice(at, at + r * c)
        nm[s] = mu * M[s] + G[s]
        nv[s] = V[s]
        u = G[s] + mu * nm[s] if nesterov else nm[s]
        new[s] = (1 - lr * wd) * P[s] - lr * max(1.0, c / r) ** 0.5 * iterate(u.view(r, c)).reshape(-1)
    keep = [x.clone() for x in d]
    out = tuple(torch.full((n,), 5.0, device=DEV) for _ in range(3))
    kw = dict(t=t, matrices=mats, nesterov=nesterov, weight_decay=wd, grad_scale=0.5)
    by_products(ctx, lambda: ctx.muon_step(*d, out=out, **kw))
    assert all(torch.equal(x, y) for x, y in zip(d, keep))
    for x, y in zip(out, (new, nm, nv)):
        assert gpu_rel(x, y) <= 1e-6
    ctx.muon_step(*d, **kw)
    assert all(torch.equal(x, y) for x, y in zip(d[:3], out))
    ctx.stats()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_bounded_wait_of_the_large_products(pkg, ctx, dtype):
    U = torch.randn(1600, 1700, generator=gen(9)).to(dtype).to(DEV)
    want = by_products(ctx, lambda: ctx.orthogonalize(U))
    ctx.set_wait_limit(2_000_000, 16)
    ctx.orthogonalize(U)
    with pytest.raises(pkg.LpError) as ei:
        ctx.stats()
    assert ei.value.status == -6
    ctx.set_wait_limit(2_000_000_000, 0)
    ctx.stats()
    assert torch.equal(ctx.orthogonalize(U), want)
    ctx.stats()


# ------------------------------------------------------------------------------------------ rows far smaller than the others
@pytest.mark.parametrize("rows,cols", [(64, 64), (128, 100), (256, 512), (1000, 300), (800, 900), (1600, 1700)])
def test_small_rows_keep_their_own_digits(ctx, rows, cols):
    """FP32: half of the rows are 1e-5 of the others.  They grow by the same factors as everything small does, and come out as near to
    64 bits, relative to themselves, as the whole matrix (2e-5).  FP32 numbers keep 24 bits of them; pairs of FP16 do only as long as
    the scales leave their low parts above 2^-24: with values of a 2048 x 2048 matrix of about 2^-11, rows of 2^-17 of that, held
    as 2^14 X, a rounding of 2^-25 is 2^-11 of them, a half of the rows' directions at random, amplified like the rows themselves."""
    U = torch.randn(rows, cols, generator=gen(rows * 5 + cols)).to(DEV)
    U[::2] *= 1e-5
    want = iterate(U)
    got = ctx.orthogonalize(U)
    assert gpu_rel(got, want) <= ORTH_TOL[F32]
    assert gpu_rel(got[::2], want[::2]) <= ORTH_TOL[F32]
    ctx.stats()


# ------------------------------------------------------------------------------------------ runs of the gradient that end at edges
@pytest.mark.parametrize("width", [33, 64, 200])     # 8, 16, 32 lanes per row: other shares of a block
@pytest.mark.parametrize("dout_t,grad_t", [(F32, F32), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("shift", [0, 1, -1])
def test_embed_grad_runs_that_end_at_edges(ctx, width, dout_t, grad_t, shift):
    """Runs of equal ids that end at (or one beside) the edges of what a group of lanes (32 ids), a span (256), a block and a block of
    joins (8,192) adds up, runs over many spans, rows named and not named on both sides of multiples of 32; into dense rows and rows
    apart.  The bound is that of the gradient: (k + 2) 2^-24 of the sum of magnitudes, and 2^-8 for a BF16 result."""
    runs = [32, 32, 192, 256, 256, 224, 1, 31, 512 - 32, 7, 249, 2048, 8192, 1, 1, 30, 224, 255, 1, 16 * 256, 17 * 256, 40 * 256, 5, 8192 - 5, 64, 3]
    runs = [max(1, r + shift * (i % 3 == 0)) for i, r in enumerate(runs)]
    named = [31, 32, 33, 63, 64, 95, 127, 128, 129, 130, 160, 191, 192, 193, 224, 255, 256, 287, 288, 319, 320, 351, 352, 383, 384, 415]
    rows = 417
    ids = torch.repeat_interleave(torch.tensor(named, dtype=torch.int32), torch.tensor(runs))
    ids = ids[torch.randperm(len(ids), generator=gen(shift + 5))].to(DEV)
    n = len(ids)
    dout = torch.randn(n, width, generator=gen(width)).to(dout_t).to(DEV)
    ref, mag = (torch.zeros(rows, width, dtype=F64, device=DEV).index_add_(0, ids.long(), 1.3 * x.double()) for x in (dout, dout.abs()))
    count = torch.bincount(ids, minlength=rows)[:, None]
    bound = (count + 2) * 2.0**-24 * mag + (ref.abs() * 2.0**-8 if grad_t == BF16 else 0.0)
    grad = torch.full((rows, width), float("nan"), dtype=grad_t, device=DEV)
    ctx.embed_grad(dout, ids, rows, scale=1.3, grad=grad)
    assert ((grad.double() - ref).abs() <= bound).all()
    assert (grad[count[:, 0] == 0] == 0).all()
    apart = torch.full((rows, width + 3), 4.0, dtype=grad_t, device=DEV)
    ctx.embed_grad(dout, ids, rows, scale=1.3, grad=apart[:, 1:width + 1])
    assert torch.equal(apart[:, 1:width + 1], grad)
    assert (apart[:, 0] == 4.0).all() and (apart[:, width + 1:] == 4.0).all()
    ctx.stats()
