"""Products with one weight matrix per group of rows, and their weight gradients, against plain 64-bit forms.

Tolerances, derived from the arithmetic:
  BF16   products of BF16 numbers are exact in FP32; the accumulator of the matrix instructions takes K / 16 (weight gradient: rows / 16,
         in blocks that are added in FP32) additions of sixteen terms, off by at most 2^-22 of the sum of magnitudes each.  Results in
         BF16 are rounded once more: 2^-8
  FP32   three BF16 parts hold 24 bits; of the nine products of parts the three smallest, 2^-7 2^-15 twice and 2^-15 2^-15, are left
         out: 2^-21 of a product at most.  A block of 64 terms takes 24 such additions, of which those of the first twenty are at most
         2^-6 of the sum, the blocks are added in FP32 (2^-24 each), and so are the partial sums of shares: off by at most
         (2^-21 + 5 * 2^-22 + (blocks + 2) * 2^-24) of the sum of magnitudes
  bias   one FP32 addition; column sums: FP32 sums of n terms in any order, n 2^-24 of the sum of magnitudes
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32


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
    rows, cols = x.shape
    buf = torch.full((rows * (cols + extra) + offset + 8,), float("nan"), dtype=x.dtype, device=DEV)
    v = buf[offset:offset + rows * (cols + extra)].view(rows, cols + extra)[:, :cols]
    v.copy_(x)
    return v


def per_term(dtype, terms):
    return terms / 16 * 2.0 ** -22 + 2.0 ** -22 if dtype == BF16 else 2.0 ** -21 + 5 * 2.0 ** -22 + (terms / 64 + 3) * 2.0 ** -24


def close(got, want, mag, per, half_step=0.0):
    err = (got.double() - want).abs()
    bound = per * mag + half_step * want.abs() + 1e-37
    worst = (err / bound).max().item() if err.numel() else 0.0
    assert worst <= 1.0, f"{worst} of the bound"


def sizes_of(kind, rows, groups, g):
    """Group ends: even, ragged with empty groups, everything in one group, and leaving rows at both ends out."""
    if kind == "even":
        cut = [rows * i // groups for i in range(groups + 1)]
    elif kind == "one":
        cut = [0] * (groups // 2 + 1) + [rows] * (groups - groups // 2)
    else:
        lo, hi = (rows // 5, rows - rows // 7) if kind == "inside" else (0, rows)
        cut = [lo] + sorted(torch.randint(lo, hi + 1, (groups - 1,), generator=g).tolist()) + [hi]
    return cut


def linear64(a, bounds, b, bias, relu, trans):
    n = b.shape[1] if trans else b.shape[2]
    out, mag = (torch.zeros(a.shape[0], n, dtype=torch.float64, device=DEV) for _ in range(2))
    for g, (lo, hi) in enumerate(zip(bounds[:-1], bounds[1:])):
        w = b[g].double().T if trans else b[g].double()
        c, m = a[lo:hi].double() @ w, a[lo:hi].double().abs() @ w.abs()
        if bias is not None:
            c, m = c + bias[g].double(), m + bias[g].double().abs()
        out[lo:hi], mag[lo:hi] = torch.relu(c) if relu else c, m
    return out, mag


SHAPES = [(1, 1, 1, 1), (7, 8, 16, 3), (130, 64, 64, 4), (300, 100, 33, 5), (257, 417, 129, 2), (1000, 256, 256, 8), (511, 72, 520, 40), (2000, 1000, 264, 7), (129, 65, 1001, 70)]


@pytest.mark.parametrize("rows,k,n,groups", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("trans", [False, True])
@pytest.mark.parametrize("kind", ["even", "ragged", "one", "inside"])
def test_grouped_linear(ctx, rows, k, n, groups, dtype, trans, kind):
    g = gen(rows + k + n)
    bounds = sizes_of(kind, rows, groups, g)
    a = torch.randn(rows, k, generator=g).to(dtype).to(DEV)
    b = torch.randn(groups, *((n, k) if trans else (k, n)), generator=g).to(dtype).to(DEV)
    bias = torch.randn(groups, n, generator=g).to(DEV) if not trans else None
    offsets = torch.tensor(bounds, dtype=I32, device=DEV)
    want, mag = linear64(a, bounds, b, bias, not trans, trans)
    for extra, offset in ((0, 0), (8, 8), (3, 1)):
        out = padded(torch.full((rows, n), 7.0, dtype=dtype), extra, offset)
        got = ctx.grouped_linear(padded(a, extra, offset), offsets, b, bias=bias, relu=not trans, trans_b=trans, out=out)
        assert got is out
        inside = slice(bounds[0], bounds[-1])
        close(got[inside], want[inside], mag[inside], per_term(dtype, k), 2.0 ** -8 if dtype == BF16 else 2.0 ** -24)
        assert (got[:bounds[0]] == 7.0).all() and (got[bounds[-1]:] == 7.0).all()
    ctx.stats()


@pytest.mark.parametrize("rows,k,n,groups", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["even", "ragged", "one", "inside"])
def test_grouped_weight_grad(ctx, rows, k, n, groups, dtype, kind):
    g = gen(rows + k + n + 1)
    bounds = sizes_of(kind, rows, groups, g)
    a = torch.randn(rows, k, generator=g).to(dtype).to(DEV)
    dz = torch.randn(rows, n, generator=g).to(dtype).to(DEV)
    offsets = torch.tensor(bounds, dtype=I32, device=DEV)
    pairs = [(a[lo:hi].double(), dz[lo:hi].double()) for lo, hi in zip(bounds[:-1], bounds[1:])]
    want, mag = torch.stack([x.T @ y for x, y in pairs]), torch.stack([x.T.abs() @ y.abs() for x, y in pairs])
    want_b, mag_b = torch.stack([y.sum(0) for _, y in pairs]), torch.stack([y.abs().sum(0) for _, y in pairs])
    longest = max(hi - lo for lo, hi in zip(bounds[:-1], bounds[1:]))
    for extra, offset in ((0, 0), (8, 8), (3, 1)):
        va, vz = padded(a, extra, offset), padded(dz, extra, offset)
        dw, db = ctx.grouped_weight_grad(va, vz, offsets, bias=True)
        close(dw, want, mag, per_term(dtype, longest))
        close(db, want_b, mag_b, (longest + 1) * 2.0 ** -24)
        assert torch.equal(ctx.grouped_weight_grad(va, vz, offsets), dw)
        dw2, db2 = dw.clone(), db.clone()
        ctx.grouped_weight_grad(va, vz, offsets, accumulate=True, dW=dw2, dbias=db2)
        assert torch.equal(dw2, dw + dw) and torch.equal(db2, db + db)
    ctx.stats()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,k,n,groups", [(70_001, 256, 256, 8), (40_003, 264, 512, 3), (33_333, 417, 250, 100), (9_000, 1024, 1032, 300)])
def test_grouped_large(ctx, rows, k, n, groups, dtype):
    """Many tiles per block, tiles shared by several blocks, more groups than a warp looks at at once."""
    g = gen(rows)
    bounds = sizes_of("ragged", rows, groups, g)
    a, dz = torch.randn(rows, k, generator=g).to(dtype).to(DEV), torch.randn(rows, n, generator=g).to(dtype).to(DEV)
    b = torch.randn(groups, k, n, generator=g).to(dtype).to(DEV)
    offsets = torch.tensor(bounds, dtype=I32, device=DEV)
    want, mag = linear64(a, bounds, b, None, False, False)
    close(ctx.grouped_linear(a, offsets, b), want, mag, per_term(dtype, k), 2.0 ** -8 if dtype == BF16 else 2.0 ** -24)
    want, mag = linear64(dz, bounds, b, None, False, True)
    close(ctx.grouped_linear(dz, offsets, b, trans_b=True), want, mag, per_term(dtype, n), 2.0 ** -8 if dtype == BF16 else 2.0 ** -24)
    dw, db = ctx.grouped_weight_grad(a, dz, offsets, bias=True)
    for i, (lo, hi) in enumerate(zip(bounds[:-1], bounds[1:])):
        x, y = a[lo:hi].double(), dz[lo:hi].double()
        close(dw[i], x.T @ y, x.T.abs() @ y.abs(), per_term(dtype, hi - lo))
        close(db[i], y.sum(0), y.abs().sum(0), (hi - lo + 1) * 2.0 ** -24)
    again = ctx.grouped_weight_grad(a, dz, offsets, bias=True)
    assert torch.equal(again[0], dw) and torch.equal(again[1], db)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("k,n", [(64, 64), (72, 40), (65, 33)])
def test_rows_of_other_groups_do_not_leak(ctx, dtype, k, n):
    """NaN in rows outside the groups, in the neighbouring group's rows and in its matrix stays there."""
    a, dz, b = torch.ones(300, k, dtype=dtype, device=DEV), torch.ones(300, n, dtype=dtype, device=DEV), torch.ones(3, k, n, dtype=dtype, device=DEV)
    offsets = torch.tensor([10, 75, 201, 290], dtype=I32, device=DEV)
    for t in (a, dz):
        t[:10], t[75:201], t[290:] = float("nan"), float("nan"), float("nan")
    b[1] = float("nan")
    got = ctx.grouped_linear(a, offsets, b, out=torch.zeros(300, n, dtype=dtype, device=DEV))
    assert (got[10:75] == k).all() and (got[201:290] == k).all() and got[75:201].isnan().all() and (got[:10] == 0).all() and (got[290:] == 0).all()
    got = ctx.grouped_linear(dz, offsets, b, trans_b=True)
    assert (got[10:75] == n).all() and (got[201:290] == n).all()
    dw, db = ctx.grouped_weight_grad(a, dz, offsets, bias=True)
    assert (dw[0] == 65).all() and (dw[2] == 89).all() and dw[1].isnan().all() and (db[0] == 65).all() and (db[2] == 89).all() and db[1].isnan().all()


def test_grouped_fp32_keeps_range_and_digits(ctx):
    """Rows and columns of any size keep their digits; the largest numbers do not overflow on the way."""
    g = gen(4)
    a, b = torch.randn(200, 96, generator=g).to(DEV), torch.randn(1, 96, 64, generator=g).to(DEV)
    a *= 10.0 ** torch.linspace(-28, 15, 200, device=DEV)[:, None]
    b *= 10.0 ** torch.linspace(-8, 8, 64, device=DEV)
    offsets = torch.tensor([0, 200], dtype=I32, device=DEV)
    got = ctx.grouped_linear(a, offsets, b)
    want, mag = a.double() @ b[0].double(), a.double().abs() @ b[0].double().abs()
    normal = mag > 1e-30
    err = ((got.double() - want).abs() / mag)[normal]
    assert err.max() <= per_term(F32, 96)
    top = torch.full((1, 1), 3.4e38, device=DEV)
    assert torch.equal(ctx.grouped_linear(top, torch.tensor([0, 1], dtype=I32, device=DEV), torch.ones(1, 1, 1, device=DEV)), top)


def test_bad_offsets_are_clamped_and_reported(pkg, ctx):
    a = torch.ones(200, 64, dtype=BF16, device=DEV)
    b = torch.ones(3, 64, 64, dtype=BF16, device=DEV)
    for bad in ([0, 150, 100, 200], [-5, 50, 100, 200], [0, 50, 100, 2**31 - 1], [300, 400, 500, 600], [0, -2**31, 7, 200]):
        offsets = torch.tensor(bad, dtype=I32, device=DEV)
        out = ctx.grouped_linear(a, offsets, b, out=torch.zeros(200, 64, dtype=BF16, device=DEV))
        with pytest.raises(pkg.LpError) as e:
            ctx.stats()
        assert e.value.status == -1
        assert ((out == 64) | (out == 0)).all()
        dw = ctx.grouped_weight_grad(a, a, offsets)
        with pytest.raises(pkg.LpError):
            ctx.stats()
        assert dw.isfinite().all() and dw[:, 0, 0].sum() <= 200
        ctx.stats()  # reported once


def test_grouped_empty(ctx):
    e = torch.zeros(0, 32, device=DEV)
    zero = torch.zeros(3, dtype=I32, device=DEV)
    b = torch.ones(2, 32, 16, device=DEV)
    assert ctx.grouped_linear(e, zero, b).shape == (0, 16)
    dw, db = ctx.grouped_weight_grad(e, torch.zeros(0, 16, device=DEV), zero, bias=True)
    assert (dw == 0).all() and (db == 0).all() and dw.shape == (2, 32, 16)
    none = ctx.grouped_weight_grad(torch.ones(5, 32, device=DEV), torch.ones(5, 16, device=DEV), zero, bias=True)
    assert (none[0] == 0).all() and (none[1] == 0).all()
    out = torch.full((5, 16), 3.0, device=DEV)
    ctx.grouped_linear(torch.ones(5, 32, device=DEV), zero, b, out=out)
    assert (out == 3.0).all()
    ctx.grouped_linear(torch.ones(5, 32, device=DEV), zero[:1], b[:0], out=out)   # no groups at all
    assert (out == 3.0).all()


def test_grouped_gradients_against_differences(ctx):
    """Directional differences of sum(dz * grouped_linear) along the rows, the matrices and the bias, in FP32."""
    g = gen(6)
    a, b, bias, dz = (torch.randn(*s, generator=g).to(DEV) for s in ((150, 40), (4, 40, 24), (4, 24), (150, 24)))
    offsets = torch.tensor([0, 30, 30, 101, 150], dtype=I32, device=DEV)
    loss = lambda x, w, v: (ctx.grouped_linear(x, offsets, w, bias=v).double() * dz.double()).sum()
    da = ctx.grouped_linear(dz, offsets, b, trans_b=True)
    dw, db = ctx.grouped_weight_grad(a, dz, offsets, bias=True)
    for i, (x, dx) in enumerate(((a, da), (b, dw), (bias, db))):
        way = torch.randn(x.shape, generator=gen(20 + i)).to(DEV)
        plus, minus = ([*(t + s * way if t is x else t for t in (a, b, bias))] for s in (0.5, -0.5))
        diff, slope = loss(*plus) - loss(*minus), (dx.double() * way.double()).sum()
        # the map is linear in each: only rounding, 2^-19 of the sum of magnitudes of 3600 values of size 10
        assert (diff - slope).abs() < 2.0 ** -19 * 3600 * 10


def test_grouped_streams_and_graphs(pkg):
    stream = torch.cuda.Stream()
    c = pkg.Context(0, stream)
    g = gen(7)
    a, dz = torch.randn(5000, 128, generator=g).to(BF16).to(DEV), torch.randn(5000, 256, generator=g).to(BF16).to(DEV)
    b = torch.randn(5, 128, 256, generator=g).to(BF16).to(DEV)
    offsets = torch.tensor(sizes_of("ragged", 5000, 5, g), dtype=I32, device=DEV)
    y, (dw, db) = c.grouped_linear(a, offsets, b), c.grouped_weight_grad(a, dz, offsets, bias=True)   # from another current stream
    out = [torch.zeros_like(t) for t in (y, dw, db)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        c.grouped_linear(a, offsets, b, out=out[0])
        c.grouped_weight_grad(a, dz, offsets, dW=out[1], dbias=out[2])
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(out, (y, dw, db)))
    # the sizes of the groups are read on the device: a replay follows them
    offsets.copy_(torch.tensor([0, 0, 1, 2500, 4999, 5000], dtype=I32))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0], c.grouped_linear(a, offsets, b)) and torch.equal(out[1], c.grouped_weight_grad(a, dz, offsets))
    c.stats()
    del graph
    c.close()


def test_grouped_refusals(pkg, ctx):
    a, b, off = torch.zeros(6, 16, device=DEV), torch.zeros(2, 16, 8, device=DEV), torch.tensor([0, 3, 6], dtype=I32, device=DEV)
    dz = torch.zeros(6, 8, device=DEV)
    bad = [lambda: ctx.grouped_linear(a, off.long(), b), lambda: ctx.grouped_linear(a, off.cpu(), b), lambda: ctx.grouped_linear(a, off[:2], b),
           lambda: ctx.grouped_linear(a, off, b.bfloat16()), lambda: ctx.grouped_linear(a, off, b, trans_b=True), lambda: ctx.grouped_linear(a, off, b[:, :15]),
           lambda: ctx.grouped_linear(a, off, b, bias=torch.zeros(8, device=DEV)), lambda: ctx.grouped_linear(a, off, b, out=a), lambda: ctx.grouped_linear(a.half(), off, b.half()),
           lambda: ctx.grouped_linear(a.T, off, b), lambda: ctx.grouped_linear(a.cpu(), off, b), lambda: ctx.grouped_linear(a, off[:0], b[:0]),
           lambda: ctx.grouped_weight_grad(a, dz[:5], off), lambda: ctx.grouped_weight_grad(a, dz.bfloat16(), off), lambda: ctx.grouped_weight_grad(a, dz, off, accumulate=True),
           lambda: ctx.grouped_weight_grad(a, dz, off, dW=torch.zeros(2, 16, 7, device=DEV)), lambda: ctx.grouped_weight_grad(a, dz, off, dbias=torch.zeros(2, 8, dtype=BF16, device=DEV))]
    for i, call in enumerate(bad):
        with pytest.raises(pkg.LpError) as e:
            call()
        assert e.value.status == -1, i
    assert ctx.grouped_linear(a, off, b).shape == (6, 8)


def test_grouped_wait_that_runs_out(pkg):
    """The operands' wait expires (16 bytes more are expected than are copied): reported once, and the context goes on."""
    c = pkg.Context(0)
    a, b = torch.randn(1000, 128, device=DEV).bfloat16(), torch.randn(3, 128, 128, device=DEV).bfloat16()
    off = torch.tensor([0, 100, 700, 1000], dtype=I32, device=DEV)
    want, dw = c.grouped_linear(a, off, b), c.grouped_weight_grad(a, a, off, bias=True)
    c.stats()
    for call in (lambda: c.grouped_linear(a, off, b), lambda: c.grouped_weight_grad(a, a, off, bias=True)):
        c.set_wait_limit(2_000_000, 16)
        call()
        with pytest.raises(pkg.LpError) as e:
            c.stats()
        assert e.value.status == -6
        c.set_wait_limit(2_000_000_000, 0)
        c.stats()
        again = c.grouped_weight_grad(a, a, off, bias=True)
        assert torch.equal(c.grouped_linear(a, off, b), want) and torch.equal(again[0], dw[0]) and torch.equal(again[1], dw[1])
    c.close()
