"""Edges of the residual-block operators and the products by group: what a call may meet beside the cases of their own tests.

Tolerances of the products are derived in the docstring of test_gpu_grouped, those of the norms in test_gpu_blocks.
"""
import ctypes

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


@pytest.mark.parametrize("n", [16, 48, 100, 112, 1000])
def test_fp32_results_of_whole_and_short_tiles(ctx, n):
    """Results leave by TMA where a warp has all 32 rows and row by row where it does not, sixteen columns at a time out of two areas
    in turn: odd numbers of such pieces, and short tiles after whole ones.  One block of terms, so that tiles follow one another fast."""
    g = gen(n)
    sizes = [256, 130, 1, 128, 300, 127, 64, 128, 31, 200, 33] * 300
    rows, groups, k = sum(sizes), len(sizes), 64
    offsets = torch.tensor([0] + sizes).cumsum(0)
    a = torch.randn(rows, k, generator=g).to(DEV)
    b = torch.randn(3, k, n, generator=g).to(DEV)[torch.arange(groups, device=DEV) % 3]
    group = torch.repeat_interleave(torch.arange(groups), torch.tensor(sizes)).to(DEV) % 3
    want, mag = torch.empty(rows, n, dtype=torch.float64, device=DEV), torch.empty(rows, n, dtype=torch.float64, device=DEV)
    for i in range(3):
        pick = group == i
        want[pick], mag[pick] = a[pick].double() @ b[i].double(), a[pick].double().abs() @ b[i].double().abs()
    off = offsets.to(I32).to(DEV)
    first = ctx.grouped_linear(a, off, b)
    per = 2.0 ** -21 + 5 * 2.0 ** -22 + (k / 64 + 3) * 2.0 ** -24
    assert ((first.double() - want).abs() <= per * mag + 2.0 ** -24 * want.abs()).all()
    for _ in range(20):
        assert torch.equal(ctx.grouped_linear(a, off, b, out=torch.zeros_like(first)), first)


def test_two_threads_with_rows_of_different_widths(pkg):
    """Two contexts on two host threads call the same kernel with different amounts of shared memory, without anything between the calls."""
    import threading
    failed, streams = [], [torch.cuda.Stream() for _ in range(2)]
    contexts = [pkg.Context(0, s) for s in streams]

    def calls(c, x, branch):
        desc = pkg.ResidualDesc(rows=2, width=x.shape[1], stream_prec=pkg.LP_FP32, prec=pkg.LP_FP32, pre_norm=pkg.LP_NORM_RMS, eps=1e-6, scale=1.0)
        n, y, ld = torch.empty_like(x), torch.empty_like(x), x.shape[1]
        args = (c.h, ctypes.addressof(desc), x.data_ptr(), ld, x.data_ptr() if branch else None, ld, y.data_ptr() if branch else None, ld, n.data_ptr(), ld)
        f = c.lib.lp_residual_norm
        for i in range(40000):
            if f(*args) != 0:
                failed.append(c.lib.lp_last_error(c.h).decode())
                return
            if i % 500 == 499:
                c.stream.synchronize()

    torch.cuda.synchronize()
    x = [torch.randn(2, width, device=DEV) for width in (8192, 2304)]
    threads = [threading.Thread(target=calls, args=a) for a in ((contexts[0], x[0], True), (contexts[1], x[1], False))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for c in contexts:
        c.close()
    assert not failed, failed


@pytest.mark.parametrize("rows,k,n,trans", [(70, 65_536, 100, False), (1200, 65_536, 2000, False), (1200, 32_768, 2000, True), (33, 1 << 20, 8, False), (300, 2_049, 264, True), (9500, 513, 256, False)])
def test_bf16_products_of_many_terms(ctx, rows, k, n, trans):
    """Sums of one sign: every addition to the accumulator of the matrix instructions rounds towards zero, so a long one drifts.  It takes
    512 terms: 32 additions of sixteen terms, off by at most 2^-22 of the sum each, and these sums are added in FP32, 2^-24 each: the
    FP32 sum s lies within want (1 +- sums).  Rounding to BF16 is monotonic, so the result lies between the roundings of the two ends.
    (The mean of the errors says nothing: these sums differ by less than a step of BF16, so their roundings are not spread evenly.)"""
    g = torch.Generator(device=DEV).manual_seed(rows + k)
    a = torch.rand(rows, k, generator=g, device=DEV).to(BF16)
    b = torch.rand(2, *((n, k) if trans else (k, n)), generator=g, device=DEV).to(BF16)
    cut = rows // 3
    got = ctx.grouped_linear(a, torch.tensor([0, cut, rows], dtype=I32, device=DEV), b, trans_b=trans).double()
    want = torch.cat([x.double() @ (w.double().T if trans else w.double()) for x, w in ((a[:cut], b[0]), (a[cut:], b[1]))])
    sums = 32 * 2.0 ** -22 + (k / 512 + 1) * 2.0 ** -24
    low, high = ((want * (1 + way)).to(BF16).double() for way in (-sums, sums))
    assert (got >= low).all() and (got <= high).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,k,n,extra", [(3000, 256, 64, 0), (3000, 250, 301, 1), (9000, 512, 520, 0)])
def test_workspace_is_what_the_header_says(pkg, dtype, rows, k, n, extra):
    size, up = 4 if dtype == F32 else 2, lambda cols, step: -(-cols // step) * step
    a, dz = (torch.randn(rows, d + extra, device=DEV).to(dtype)[:, :d] for d in (k, n))
    b = torch.randn(3, k, n, device=DEV).to(dtype)
    off = torch.tensor([0, 100, 700, rows], dtype=I32, device=DEV)
    aligned = lambda t: t.data_ptr() % 16 == 0 and t.stride(-2) * size % 16 == 0
    copy = lambda t, cols, count: 0 if aligned(t) else up(cols, 16 // size) * size * count
    places = 2 * 256   # of at most two operands, each rounded up to 256 bytes

    def taken(call):
        c = pkg.Context(0)
        call(c)
        torch.cuda.synchronize()
        bytes_ = c.stats().workspace_bytes
        c.close()
        return bytes_

    linear = 6 * up(n, 8) * 3 * k + copy(a, k, rows) if dtype == F32 else copy(a, k, rows) + copy(b, n, 3 * k)
    assert linear <= taken(lambda c: c.grouped_linear(a, off, b)) <= linear + places
    grad = 6 * up(k, 8) * rows + copy(dz, n, rows) if dtype == F32 else copy(a, k, rows) + copy(dz, n, rows)
    assert grad <= taken(lambda c: c.grouped_weight_grad(a, dz, off, bias=True)) <= grad + places + 40_000_000


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_products_into_their_own_operands_are_refused(pkg, ctx, dtype):
    off = torch.tensor([0, 30, 100], dtype=I32, device=DEV)
    buf = torch.randn(140, 200, device=DEV).to(dtype)
    a, b = buf[:100, :64], torch.randn(2, 64, 64, device=DEV).to(dtype)
    flat = buf.view(-1)
    f32 = torch.randn(3 * 64 * 64 + 100, device=DEV)
    bad = [lambda: ctx.grouped_linear(a, off, b, out=a), lambda: ctx.grouped_linear(a, off, b, out=buf[:100, 63:127]), lambda: ctx.grouped_linear(a, off, b, out=buf[1:101, :64]),
           lambda: ctx.grouped_linear(buf[1:101, 100:164], off, b, out=buf[:100, 40:104]), lambda: ctx.grouped_linear(a, off, b, out=flat[99 * 200:99 * 200 + 6400].view(100, 64)),
           lambda: ctx.grouped_linear(a, off, flat[:2 * 64 * 64].view(2, 64, 64), out=buf[20:120, 100:164])]
    if dtype == F32:
        w = f32[:2 * 64 * 64].view(2, 64, 64)
        x = f32[4096:4096 + 6400].view(100, 64)
        bad += [lambda: ctx.grouped_weight_grad(x, a, off, dW=w), lambda: ctx.grouped_weight_grad(a, x, off, dW=w), lambda: ctx.grouped_linear(a, off, b, bias=w.view(-1)[:128].view(2, 64), out=f32[100:6500].view(100, 64)),
                lambda: ctx.grouped_weight_grad(a, a, off, dW=w, dbias=f32[100:228].view(2, 64)), lambda: ctx.grouped_weight_grad(a, x, off, dW=torch.zeros_like(w), dbias=f32[4100:4228].view(2, 64))]
    for i, call in enumerate(bad):
        with pytest.raises(pkg.LpError) as e:
            call()
        assert e.value.status == -1, i
    # beside one another in one buffer, and behind one another
    want = ctx.grouped_linear(a, off, b)
    assert torch.equal(ctx.grouped_linear(a, off, b, out=buf[:100, 64:128]), want)
    assert torch.equal(ctx.grouped_linear(a, off, b, out=buf[:100, 136:200]), want)
    assert torch.equal(ctx.grouped_linear(a, off, b, out=flat[99 * 200 + 64:99 * 200 + 64 + 6400].view(100, 64)), want)
    one = ctx.grouped_linear(a[:1], torch.tensor([0, 0, 1], dtype=I32, device=DEV), b)
    assert torch.equal(ctx.grouped_linear(buf[:1, :64], torch.tensor([0, 0, 1], dtype=I32, device=DEV), b, out=buf[:1, 64:128]), one)


def test_overlapping_results_of_dropout_and_norms_are_refused(pkg, ctx):
    buf, w = torch.randn(70, 200, device=DEV), torch.ones(64, device=DEV)
    x, h, z = buf[:60, :64], buf[:60, 64:128], torch.randn(60, 64, device=DEV)
    shifted, beside = buf[1:61, :64], buf[:60, 128:192]
    half = z.view(BF16).view(60, 128)[:, :64]          # the same memory as another type
    bad = [lambda: ctx.dropout(x, 0.5, 1, 1, out=shifted), lambda: ctx.dropout(x, 0.5, 1, 1, out=buf[:60, 1:65]), lambda: ctx.dropout(z, 0.5, 1, 1, out=z.view(-1)[8:8 + 58 * 64].view(58, 64)),
           lambda: ctx.residual_norm(x, h, y=shifted), lambda: ctx.residual_norm(x, h, n=buf[:60, 65:129]), lambda: ctx.residual_norm(x, h, y=z, n=z), lambda: ctx.residual_norm(z, dtype=BF16, n=half),
           lambda: ctx.residual_norm(z, gate=w, h=h, pre=z.view(-1)[:64], y=z), lambda: ctx.residual_norm_grad(x, h, z, z, dx=shifted), lambda: ctx.residual_norm_grad(x, h, z, z, dx=beside, dh=beside),
           lambda: ctx.residual_norm_grad(x, h, z, z, pre=w, dpre=z.view(-1)[:64]), lambda: ctx.residual_norm_grad(x, h, z, z, pre=w, post_norm="rms", post=w, dpre=beside[0], dpost=beside[0]),
           lambda: ctx.residual_norm_grad(x, h, z, z, gate=w, dgate=w[:64], pre=w, dpre=w)]
    before = buf.clone(), z.clone()
    for i, call in enumerate(bad):
        with pytest.raises(pkg.LpError) as e:
            call()
        assert e.value.status == -1, i
    assert torch.equal(buf, before[0]) and torch.equal(z, before[1])
    y, n = ctx.residual_norm(x, h)
    got = ctx.residual_norm(x, h, y=beside, n=torch.empty(60, 64, device=DEV))
    assert torch.equal(got[0], y) and torch.equal(got[1], n)
    a, b = x.clone(), h.clone()                          # results in each other's inputs' places
    got = ctx.residual_norm(a, b, y=b, n=a)
    assert torch.equal(got[0], y) and torch.equal(got[1], n)
    want = ctx.residual_norm_grad(z, x, y, h)
    dn, yy = x.clone(), y.clone()
    got = ctx.residual_norm_grad(z, dn, yy, h, dx=dn, dh=yy)
    assert torch.equal(got["dx"], want["dx"]) and torch.equal(got["dh"], want["dh"])
    drop = ctx.dropout(x, 0.5, 1, 1)
    assert torch.equal(ctx.dropout(x, 0.5, 1, 1, out=beside), drop) and torch.equal(ctx.dropout(x, 0.5, 1, 1, out=x), drop)


def test_scales_beyond_fp32_are_refused(pkg, ctx):
    x = torch.ones(4, 16, device=DEV)
    for scale, p in ((1e39, 0.0), (-1e300, 0.0), (3e38, 0.5), (1e300, 1.0), (float("inf"), 0.0), (float("nan"), 0.1)):
        for call in (lambda: ctx.residual_norm(x, x, scale=scale, p=p), lambda: ctx.residual_norm_grad(x, x, x, x, scale=scale, p=p)):
            with pytest.raises(pkg.LpError) as e:
                call()
            assert e.value.status == -1
    y, _ = ctx.residual_norm(x, x, scale=3e38)
    assert (y == torch.tensor(3e38)).all() and (ctx.residual_norm(x, x, scale=3e38, p=1.0)[0] == 1.0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_batches_without_rows_and_without_a_norm_before_the_next_block(ctx, dtype):
    x, h, w = torch.zeros(0, 48, device=DEV), torch.zeros(0, 48, dtype=dtype, device=DEV), torch.full((48,), 3.0, device=DEV)
    y, n = ctx.residual_norm(x, h, pre_norm=None)
    assert y.shape == (0, 48) and n is None
    assert ctx.residual_norm(x, h, pre_norm=None, post_norm="rms", post=w, gate=h)[0].shape == (0, 48)
    got = ctx.residual_norm_grad(x, None, x, h, pre_norm=None)
    assert set(got) == {"dx", "dh"} and got["dh"].dtype == dtype
    got = ctx.residual_norm_grad(x, None, x, h, pre_norm=None, gate=h)
    assert got["dgate"].shape == (0, 48)
    got = ctx.residual_norm_grad(x, None, x, h, pre_norm=None, post_norm="layer", post=w, post_bias=w, gate=w)
    assert all((got[k] == 0).all() and got[k].shape == (48,) for k in ("dpost", "dpost_bias", "dgate"))
    ctx.residual_norm_grad(x, None, x, h, pre_norm=None, post_norm="layer", post=w, dpost=w, accumulate=True)
    assert (w == 3.0).all()


def test_parameters_of_norms_that_are_not_taken(pkg, ctx):
    """They change nothing forward and have no gradient; asking for one by name is refused."""
    x, h, dy = (torch.randn(30, 40, generator=gen(s)).to(DEV) for s in (1, 2, 3))
    w, params = torch.full((40,), 2.0, device=DEV), ("pre", "pre_bias", "post", "post_bias")
    every = {k: w for k in params}
    assert torch.equal(ctx.residual_norm(x, h, pre_norm=None, **every)[0], ctx.residual_norm(x, h, pre_norm=None)[0])
    got, want = ctx.residual_norm_grad(dy, None, x, h, pre_norm=None, **every), ctx.residual_norm_grad(dy, None, x, h, pre_norm=None)
    assert set(got) == set(want) == {"dx", "dh"} and all(torch.equal(got[k], want[k]) for k in want)
    # before the first block there is only the norm before it
    assert torch.equal(ctx.residual_norm(x, post_norm="rms", gate=w, **every)[1], ctx.residual_norm(x, pre=w, pre_bias=w)[1])
    got, want = ctx.residual_norm_grad(dy, h, x, post_norm="rms", gate=w, **every), ctx.residual_norm_grad(dy, h, x, pre=w, pre_bias=w)
    assert set(got) == set(want) == {"dx", "dpre", "dpre_bias"} and all(torch.equal(got[k], want[k]) for k in want)
    for kw in (dict(pre_norm=None, dpre=w), dict(pre_norm=None, dpost_bias=w)):
        with pytest.raises(pkg.LpError) as e:
            ctx.residual_norm_grad(dy, None, x, h, **kw)
        assert e.value.status == -1


def test_bad_ids_and_bad_offsets_are_both_reported(pkg):
    c = pkg.Context(0)
    table, a, b = torch.ones(5, 16, device=DEV), torch.ones(4, 16, device=DEV), torch.ones(1, 16, 16, device=DEV)
    for order in (0, 1):
        calls = [lambda: c.embed(table, torch.tensor([1, 9], dtype=I32, device=DEV)), lambda: c.grouped_linear(a, torch.tensor([3, 1], dtype=I32, device=DEV), b)]
        for call in calls[::-1] if order else calls:
            call()
        said = []
        for _ in range(2):
            with pytest.raises(pkg.LpError) as e:
                c.stats()
            assert e.value.status == -1
            said.append(str(e.value))
        assert sorted("offsets" in s for s in said) == [False, True] and sorted("id outside" in s for s in said) == [False, True]
        c.stats()
    c.close()


@pytest.mark.parametrize("dtype,rows,k,n,size", [(BF16, 9500, 256, 256, 1900), (BF16, 9500, 256, 256, 30), (BF16, 9500, 1024, 512, 700), (F32, 3000, 128, 128, 600), (F32, 3000, 200, 300, 30), (F32, 3001, 1024, 129, 100),
                                                 (BF16, 700, 1024, 96, 50)])
def test_waits_of_every_kind_of_product_that_run_out(pkg, dtype, rows, k, n, size):
    """The operands' wait of one block expires (16 bytes more are announced than come): pairs of blocks, operands that are split on their
    way, accumulators in turn, groups that end within the first block of rows.  Reported once, and the context goes on."""
    c = pkg.Context(0)
    g = gen(rows + k)
    bounds = list(range(0, rows, size)) + [rows]
    groups = len(bounds) - 1
    a, dz = torch.randn(rows, k, generator=g).to(dtype).to(DEV), torch.randn(rows, n, generator=g).to(dtype).to(DEV)
    b = torch.randn(groups, k, n, generator=g).to(dtype).to(DEV)
    off = torch.tensor(bounds, dtype=I32, device=DEV)
    calls = (lambda: [c.grouped_linear(a, off, b)], lambda: [c.grouped_linear(dz, off, b, trans_b=True)], lambda: [*c.grouped_weight_grad(a, dz, off, bias=True)], lambda: [c.grouped_weight_grad(a, dz, off)])
    want = [call() for call in calls]
    c.stats()
    for call in calls:
        c.set_wait_limit(2_000_000, 16)
        call()
        with pytest.raises(pkg.LpError) as e:
            c.stats()
        assert e.value.status == -6
        c.set_wait_limit(2_000_000_000, 0)
        c.stats()
        for again, first in zip(calls, want):
            assert all(torch.equal(x, y) for x, y in zip(again(), first))
    c.stats()
    c.close()


@pytest.mark.parametrize("width", [1040, 1041])
def test_residual_norm_offsets_beyond_32_bits(ctx, width):
    """Rows do not depend on one another: those at both ends of 4.4e9 elements have the bits of a call of their own."""
    rows = (1 << 22) + 3
    g = torch.Generator(device=DEV).manual_seed(width)
    x, h = (torch.empty(rows, width, dtype=BF16, device=DEV) for _ in range(2))
    ends = [slice(0, 3), slice(rows // 2, rows // 2 + 2), slice(rows - 5, rows)]
    for t in (x, h):
        t.fill_(0.5)
        for e in ends:
            t[e].normal_(generator=g)
    w = 1 + 0.1 * torch.randn(width, generator=g, device=DEV)
    args = dict(pre=w, post_norm="layer", post=w, gate=w, scale=0.5, p=0.3, seed=5, step=6)
    small = [(x[e].clone(), h[e].clone()) for e in ends]
    want = [ctx.residual_norm(a, b, row_base=e.start, **args) for (a, b), e in zip(small, ends)]
    y, n = ctx.residual_norm(x, h, **args)
    for (wy, wn), e in zip(want, ends):
        assert torch.equal(y[e], wy) and torch.equal(n[e], wn)
    grads = [ctx.residual_norm_grad(a, b, wy, b, row_base=e.start, **args) for (a, b), (wy, _), e in zip(small, want, ends)]
    got = ctx.residual_norm_grad(x, h, y, h, dx=x, dh=n, **args)
    for first, e in zip(grads, ends):
        assert torch.equal(got["dx"][e], first["dx"]) and torch.equal(got["dh"][e], first["dh"])
    del x, h, y, n, got
    torch.cuda.empty_cache()


def products_close(got, a, w, dtype, terms):
    want, mag = a.double() @ w.double(), a.double().abs() @ w.double().abs()
    per = terms / 16 * 2.0 ** -22 + 2.0 ** -22 if dtype == BF16 else 2.0 ** -21 + 5 * 2.0 ** -22 + (terms / 64 + 3) * 2.0 ** -24
    assert ((got.double() - want).abs() <= per * mag + (2.0 ** -8 if got.dtype == BF16 else 2.0 ** -24) * want.abs()).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("k", [520, 521])
def test_products_of_rows_beyond_32_bits(ctx, dtype, k):
    rows, n = (1 << 22) + 3, 520
    a = torch.randn(rows, k, dtype=dtype, device=DEV)
    b = torch.randn(3, k, n, device=DEV).to(dtype)
    bounds = [0, 1000, rows - 900, rows]
    off = torch.tensor(bounds, dtype=I32, device=DEV)
    c = ctx.grouped_linear(a, off, b)
    for part, i in ((slice(0, 300), 0), (slice(rows - 1300, rows - 900), 1), (slice(rows - 900, rows), 2)):
        products_close(c[part], a[part], b[i], dtype, k)
    dw = ctx.grouped_weight_grad(a, c, off)
    for part, i in ((slice(0, 1000), 0), (slice(rows - 900, rows), 2)):
        products_close(dw[i], a[part].T, c[part], dtype, 1000)
    del a, c
    torch.cuda.empty_cache()
    ctx.stats()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [2048, 2047])
def test_products_with_matrices_beyond_32_bits(ctx, dtype, n):
    groups, k, each = 520, 2048, 12
    b = torch.randn(groups, k, n, dtype=dtype, device=DEV)
    a, dz = (torch.randn(groups * each, d, device=DEV).to(dtype) for d in (k, n))
    off = torch.arange(groups + 1, dtype=I32, device=DEV) * each
    c, da = ctx.grouped_linear(a, off, b), ctx.grouped_linear(dz, off, b, trans_b=True)
    dw, db = ctx.grouped_weight_grad(a, dz, off, bias=True)
    assert b.numel() > 1 << 31 and dw.numel() > 1 << 31
    for i in (0, 1, groups - 9, groups - 1):
        part = slice(i * each, (i + 1) * each)
        products_close(c[part], a[part], b[i], dtype, k)
        products_close(da[part], dz[part], b[i].T, dtype, n)
        products_close(dw[i], a[part].T, dz[part], dtype, each)
        assert ((db[i].double() - dz[part].double().sum(0)).abs() <= (each + 1) * 2.0 ** -24 * dz[part].double().abs().sum(0)).all()
    del b, dw
    torch.cuda.empty_cache()
    ctx.stats()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("groups,rows,k,n", [(5_000, 40_000, 72, 40), (100_000, 60_000, 24, 16), (1 << 20, 30_000, 8, 8)])
def test_very_many_groups(ctx, dtype, groups, rows, k, n):
    """Up to the largest number of groups, most of them of a few rows or none."""
    g = gen(groups)
    bounds = torch.cat((torch.tensor([0]), torch.randint(0, rows + 1, (groups - 1,), generator=g).sort().values, torch.tensor([rows])))
    a, dz = torch.randn(rows, k, generator=g).to(dtype).to(DEV), torch.randn(rows, n, generator=g).to(dtype).to(DEV)
    b = torch.randn(groups, k, n, device=DEV).to(dtype)
    off = bounds.to(I32).to(DEV)
    group = torch.repeat_interleave(torch.arange(groups), bounds.diff()).to(DEV)
    w = b[group].double()
    want, mag = torch.einsum("rk,rkn->rn", a.double(), w), torch.einsum("rk,rkn->rn", a.double().abs(), w.abs())
    per = lambda terms: terms / 16 * 2.0 ** -22 + 2.0 ** -22 if dtype == BF16 else 2.0 ** -21 + 5 * 2.0 ** -22 + (terms / 64 + 3) * 2.0 ** -24
    got = ctx.grouped_linear(a, off, b)
    assert ((got.double() - want).abs() <= per(k) * mag + (2.0 ** -8 if dtype == BF16 else 2.0 ** -24) * want.abs()).all()
    dw, db = ctx.grouped_weight_grad(a, dz, off, bias=True)
    outer = a.double()[:, :, None] * dz.double()[:, None, :]
    want = torch.zeros(groups, k, n, dtype=torch.float64, device=DEV).index_add_(0, group, outer)
    mag = torch.zeros(groups, k, n, dtype=torch.float64, device=DEV).index_add_(0, group, outer.abs())
    longest = int(bounds.diff().max())
    assert ((dw.double() - want).abs() <= per(longest) * mag).all()
    want = torch.zeros(groups, n, dtype=torch.float64, device=DEV).index_add_(0, group, dz.double())
    mag = torch.zeros(groups, n, dtype=torch.float64, device=DEV).index_add_(0, group, dz.double().abs())
    assert ((db.double() - want).abs() <= (longest + 1) * 2.0 ** -24 * mag).all()
    ctx.stats()


def block_of_calls(c, dtype, rows, width, seed):
    """Inputs, and a function that runs a whole block and its gradients into given results (or new ones)."""
    g = gen(seed)
    x, dy = (torch.randn(rows, width, generator=g).to(DEV) for _ in range(2))
    w = (1 + 0.1 * torch.randn(width, generator=g)).to(DEV)
    b, bias = torch.randn(5, width, width, generator=g).to(dtype).to(DEV), torch.randn(5, width, generator=g).to(DEV)
    off = torch.tensor([0, rows // 7, rows // 7, rows // 2, rows - 3, rows], dtype=I32, device=DEV)
    args = dict(pre=w, post_norm="rms", post=w, gate=w, scale=0.5, p=0.2, seed=seed, step=4)

    def run(o=None):
        o = o or {}
        n = c.dropout(x.to(dtype), 0.1, seed, 5, out=o.get("n"))
        h = c.grouped_linear(n, off, b, bias=bias, relu=True, out=o.get("h"))
        y, m = c.residual_norm(x, h, y=o.get("y"), n=o.get("m"), **args)
        d = c.residual_norm_grad(dy, m, y, h, **{k: o.get(k) for k in ("dx", "dh", "dpre", "dpost", "dgate")}, **args)
        da = c.grouped_linear(d["dh"], off, b, trans_b=True, out=o.get("da"))
        dw, db = c.grouped_weight_grad(n, d["dh"], off, bias=True, dW=o.get("dw"), dbias=o.get("db"))
        return dict(n=n, h=h, y=y, m=m, da=da, dw=dw, db=db, **d)

    return off, run


@pytest.mark.parametrize("dtype,rows,width", [(BF16, 10_000, 256), (F32, 3_000, 192), (BF16, 3_001, 100)])
def test_two_captured_blocks_share_a_workspace(pkg, dtype, rows, width):
    """Pairs of blocks and FP32 operands too; replayed in turn, with groups that change between replays."""
    stream = torch.cuda.Stream()
    c = pkg.Context(0, stream)
    with torch.cuda.stream(stream):
        calls = [block_of_calls(c, dtype, r, width, s) for r, s in ((rows, 1), (rows // 2, 2))]
        want = [{k: v.clone() for k, v in run().items()} for _, run in calls]
        outs = [{k: torch.zeros_like(v) for k, v in w.items()} for w in want]
        stream.synchronize()
        graphs = [torch.cuda.CUDAGraph() for _ in calls]
        for graph, out, (_, run) in zip(graphs, outs, calls):
            with torch.cuda.graph(graph, stream=stream):
                run(out)
        for _ in range(3):
            for out in outs:
                for v in out.values():
                    v.zero_()
            for graph in graphs:
                graph.replay()
            stream.synchronize()
            for out, w in zip(outs, want):
                assert all(torch.equal(out[k], w[k]) for k in w)
        off, run = calls[0]
        off.copy_(torch.tensor([0, 1, 700, 701, 701, rows], dtype=I32))
        graphs[0].replay()
        again = run()
        stream.synchronize()
        assert all(torch.equal(outs[0][k], again[k]) for k in again) and not torch.equal(again["dw"], want[0]["dw"])
    c.stats()
    del graphs
    c.close()


def test_two_contexts_at_once(pkg):
    """Two streams run whole blocks beside one another, from two host threads; each gets the bits that it gets alone."""
    import threading
    streams = [torch.cuda.Stream() for _ in range(2)]
    contexts = [pkg.Context(0, s) for s in streams]
    runs, want = [], []
    for c, s, kind in zip(contexts, streams, ((BF16, 20_000, 256, 3), (F32, 8_000, 200, 4))):
        with torch.cuda.stream(s):
            runs.append(block_of_calls(c, *kind)[1])
            want.append(runs[-1]())
            s.synchronize()
    failed = []

    def loop(i):
        try:
            with torch.cuda.stream(streams[i]):
                for _ in range(40):
                    got = runs[i]()
                    if not all(torch.equal(got[k], want[i][k]) for k in got):
                        failed.append(i)
                contexts[i].stats()
        except Exception as e:
            failed.append(e)

    threads = [threading.Thread(target=loop, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for c in contexts:
        c.close()
    assert not failed, failed


def test_refused_offsets_are_named(pkg, ctx):
    a, b = torch.zeros(4, 16, device=DEV), torch.zeros(2, 16, 16, device=DEV)
    off = torch.tensor([0, 2, 4], dtype=I32, device=DEV)
    for bad in (off.long(), off.cpu(), off[None], off[:0], torch.zeros(6, dtype=I32, device=DEV)[::2]):
        for call in (lambda: ctx.grouped_linear(a, bad, b), lambda: ctx.grouped_weight_grad(a, a, bad)):
            with pytest.raises(pkg.LpError, match="offsets"):
                call()
