"""Dropout and the residual norm, forward and backward, against plain 64-bit forms.

Tolerances, derived from the arithmetic (u = 2^-24, the rounding of one FP32 operation):
  dropout        one FP32 product and one rounding: bit for bit what the same two operations give
  norms          a row's sums are trees of at most 8 + 10 + 2 additions over products rounded once, so they are off by at most 21 u of
                 the sum of their terms' magnitudes; 1 / sqrt halves that and adds 3 u; the mean of a layer norm is off by 21 u of the
                 mean magnitude, which counts |mean| r times more after the division by the standard deviation.  Products and sums
                 after that: fewer than 16 further roundings.  So an element is off by at most 64 u times the sum of the magnitudes
                 of the terms that it is made of (`mag`, formed in 64 bits with every term's magnitude), and the weights in `mag` of
                 a layer norm carry the factor 1 + |mean| r
  BF16 results   one rounding more: 2^-8 of the value
  column sums    FP32 sums of N terms in any order: N u of the terms' magnitudes on top of each term's own 64 u
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F64 = torch.float32, torch.bfloat16, torch.float64
U = 2.0 ** -24
HALF_STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


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


def philox(ctr, key):
    """Philox4x32-10 on uint64 arrays holding 32-bit words."""
    c0, c1, c2, c3 = (np.asarray(c, dtype=np.uint64) for c in ctr)
    k0, k1 = key
    m32 = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c0 * np.uint64(0xD2511F53), c2 * np.uint64(0xCD9E8D57)
        c0, c1, c2, c3 = (b >> np.uint64(32)) ^ c1 ^ np.uint64(k0), b & m32, (a >> np.uint64(32)) ^ c3 ^ np.uint64(k1), a & m32
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c0, c1, c2, c3


def keep_mask(rows, width, p, seed, step, row_base=0):
    t = int(round(65536 * p))
    groups = (width + 7) // 8
    r = (np.arange(rows, dtype=np.uint64) + np.uint64(row_base))[:, None] + np.zeros((1, groups), np.uint64)
    g = np.arange(groups, dtype=np.uint64)[None, :] + np.zeros((rows, 1), np.uint64)
    w = philox((r & np.uint64(0xFFFFFFFF), r >> np.uint64(32), np.full_like(r, step & 0xFFFFFFFF), np.uint64(5) | g << np.uint64(8)),
               (seed & 0xFFFFFFFF, seed >> 32))
    u = np.stack([h for x in w for h in (x & np.uint64(0xFFFF), x >> np.uint64(16))], axis=-1).reshape(rows, groups * 8)[:, :width]
    return torch.from_numpy(u >= np.uint64(t)), (65536.0 / (65536 - t) if t < 65536 else 0.0)


# ------------------------------------------------------------------------------------------ dropout
@pytest.mark.parametrize("rows,width", [(1, 1), (3, 7), (5, 8), (70, 64), (33, 100), (257, 417), (9, 2049), (1000, 256), (2, 70001)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("extra,offset", [(0, 0), (8, 0), (1, 1)])
def test_dropout_bits(ctx, rows, width, dtype, extra, offset):
    x = torch.randn(rows, width, generator=gen(rows + width)).to(dtype)
    seed, step = (rows << 40) + width + 77, (1 << 35) + 5
    for p in (0.1, 0.5):
        keep, factor = keep_mask(rows, width, p, seed, step)
        want = torch.where(keep, (x.float() * np.float32(factor)).to(dtype), torch.zeros((), dtype=dtype))
        got = ctx.dropout(padded(x, extra, offset), p, seed, step)
        assert torch.equal(got.cpu(), want)
        out = padded(torch.zeros(rows, width, dtype=dtype), extra, offset)
        ctx.dropout(x.to(DEV), p, seed, step, out=out)
        assert torch.equal(out.cpu(), want)
        ctx.dropout(out, 0.0, seed, step, out=out)
        assert torch.equal(out.cpu(), want)


def test_dropout_rate_and_edges(ctx):
    x = torch.ones(4000, 250, device=DEV)
    for p in (0.05, 0.3, 0.9):
        got = ctx.dropout(x, p, seed=9, step=1)
        share = (got == 0).double().mean().item()
        assert abs(share - p) < 6 * (p * (1 - p) / x.numel()) ** 0.5 + 2.0 ** -17   # six standard deviations and the rounding of p
    x[3, 5], x[4, 6] = float("nan"), float("inf")
    assert (ctx.dropout(x, 1.0, 9, 1) == 0).all()
    assert torch.equal(ctx.dropout(x, 0.0, 9, 1).nan_to_num(7.0), x.nan_to_num(7.0))
    keep, _ = keep_mask(4000, 250, 0.5, 9, 1)
    got = ctx.dropout(x, 0.5, 9, 1).cpu()
    assert (got[~keep] == 0).all()                  # also where NaN and infinity stood
    assert ctx.dropout(x[:0], 0.5, 9, 1).shape == (0, 250)


def test_dropout_does_not_depend_on_the_split(ctx):
    x = torch.randn(1001, 96, generator=gen(3)).to(DEV)
    base = (1 << 32) - 500                          # rows on both sides of 2^32
    whole = ctx.dropout(x, 0.4, 5, 6, row_base=base)
    parts = torch.cat([ctx.dropout(x[a:b], 0.4, 5, 6, row_base=base + a) for a, b in ((0, 1), (1, 500), (500, 1001))])
    assert torch.equal(whole, parts)
    keep, factor = keep_mask(1001, 96, 0.4, 5, 6, base)
    assert torch.equal(whole.cpu() != 0, keep)
    assert not torch.equal(whole, ctx.dropout(x, 0.4, 5, 7, row_base=base)) and not torch.equal(whole, ctx.dropout(x, 0.4, 6, 6, row_base=base))


def test_dropout_offsets_beyond_32_bits(ctx):
    rows, width = (1 << 22) + 3, 1040               # 4.4e9 elements, 8.7 GB
    x = torch.ones(rows, width, dtype=BF16, device=DEV)
    ctx.dropout(x, 0.5, 1, 2, out=x)
    for r in (0, rows - 3, rows - 1):
        keep, _ = keep_mask(1, width, 0.5, 1, 2, r)
        assert torch.equal(x[r].cpu() != 0, keep[0])
    del x
    torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------ residual norm
def norm64(v, kind, w, b, eps):
    """The norm and the magnitude of what it is made of."""
    amp = torch.ones_like(v[:, :1])
    mag = v.abs()
    if kind == "layer":
        mean = v.mean(1, keepdim=True)
        mag = mag + v.abs().mean(1, keepdim=True)
        v = v - mean
    r = 1.0 / torch.sqrt(v.square().mean(1, keepdim=True) + eps)
    z = v * r
    out, mag = z * w, mag * r * w.abs() * amp
    if b is not None:
        out, mag = out + b, mag + b.abs()
    return out, mag


def case_inputs(rows, width, stream, dtype, pre_norm, post_norm, bias, gate, seed):
    g = gen(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)
    t = dict(x=(1.5 * rnd(rows, width) + 0.3).to(stream), h=(0.7 * rnd(rows, width) - 0.2).to(dtype))
    t["pre"] = 1 + 0.1 * rnd(width) if pre_norm else None
    t["post"] = 1 + 0.1 * rnd(width) if post_norm else None
    t["pre_bias"] = 0.1 * rnd(width) if pre_norm and bias else None
    t["post_bias"] = 0.1 * rnd(width) if post_norm and bias else None
    t["gate"] = 1 + 0.2 * rnd(width) if gate == "vector" else rnd(rows, width).sigmoid().to(dtype) if gate == "matrix" else None
    t["dy"], t["dn"] = 1e-3 * rnd(rows, width), 1e-3 * rnd(rows, width)
    t["dy"], t["dn"] = t["dy"].to(stream), t["dn"].to(dtype)
    return {k: v.to(DEV) if v is not None else None for k, v in t.items()}


def forward64(t, kinds, scale, keep, factor, eps):
    d = {k: v.double() if v is not None else None for k, v in t.items()}
    b, mag = d["h"], d["h"].abs()
    ones = torch.ones(b.shape[1], dtype=F64, device=DEV)
    if kinds[1]:
        b, mag = norm64(b, kinds[1], d["post"] if d["post"] is not None else ones, d["post_bias"], eps)
    b, mag = torch.where(keep, b * factor, 0.0), torch.where(keep, mag * factor, 0.0)
    if d["gate"] is not None:
        b, mag = b * d["gate"], mag * d["gate"].abs()
    y = d["x"] + scale * b
    mag = d["x"].abs() + abs(scale) * mag
    if not kinds[0]:
        return y, mag, None, None
    n, mag_n = norm64(y, kinds[0], d["pre"] if d["pre"] is not None else ones, d["pre_bias"], eps)
    # what y is off by, next to what the norm itself is off by
    r = mag_n / (mag + 1e-300)
    v = y - y.mean(1, keepdim=True) if kinds[0] == "layer" else y
    r = 1.0 / torch.sqrt(v.square().mean(1, keepdim=True) + eps)
    w = d["pre"].abs() if d["pre"] is not None else ones
    return y, mag, n, mag_n + 2 * w * r * (mag + mag.square().mean(1, keepdim=True).sqrt())


def close(got, want, mag, ulps, dtype):
    err = (got.double() - want).abs()
    bound = ulps * U * mag + HALF_STEP[dtype] * want.abs() + 1e-40
    worst = (err / bound).max().item() if err.numel() else 0.0
    assert worst <= 1.0, f"{worst} of the bound"


WIDTHS = [(1, 1), (3, 7), (65, 64), (33, 100), (257, 417), (50, 256), (64, 1000), (130, 2048), (3, 5000), (2, 8192)]
KINDS = [("rms", None, "none", 0.0), ("rms", "rms", "vector", 0.1), ("layer", "layer", "matrix", 0.25), (None, "rms", "none", 0.5), ("layer", None, "vector", 0.0),
         (None, None, "matrix", 0.3), ("layer", "layer", "vector", 0.0), ("layer", "layer", "none", 0.1)]


@pytest.mark.parametrize("rows,width", WIDTHS)
@pytest.mark.parametrize("stream,dtype", [(F32, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("pre_norm,post_norm,gate,p", KINDS)
def test_residual_norm(ctx, rows, width, stream, dtype, pre_norm, post_norm, gate, p):
    t = case_inputs(rows, width, stream, dtype, pre_norm, post_norm, "layer" in (pre_norm, post_norm), gate, rows * 31 + width)
    seed, step, scale, eps = 1234567890123, 17, -0.75, 1e-5
    keep, factor = keep_mask(rows, width, p, seed, step, 40)
    keep = keep.to(DEV)
    y64, mag_y, n64, mag_n = forward64(t, (pre_norm, post_norm), scale, keep, factor, eps)
    args = dict(pre_norm=pre_norm, post_norm=post_norm, scale=scale, p=p, seed=seed, step=step, row_base=40, eps=eps, pre=t["pre"], pre_bias=t["pre_bias"],
                post=t["post"], post_bias=t["post_bias"])
    for extra, offset in ((0, 0), (16, 8), (3, 1)):
        v = {k: padded(t[k], extra, offset) if t[k] is not None and t[k].dim() == 2 else t[k] for k in ("x", "h", "gate")}
        y, n = ctx.residual_norm(v["x"], v["h"], gate=v["gate"], **args)
        close(y, y64, mag_y, 64, stream)
        if pre_norm:
            close(n, n64, mag_n, 64, dtype)
        else:
            assert n is None
        # results over the inputs
        y2, n2 = ctx.residual_norm(v["x"], v["h"], gate=v["gate"], y=v["x"], n=v["h"] if pre_norm else None, **args)
        assert torch.equal(y2, y) and (n is None or torch.equal(n2, n))


@pytest.mark.parametrize("rows,width", WIDTHS)
@pytest.mark.parametrize("stream,dtype", [(F32, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("pre_norm,post_norm,gate,p", KINDS)
def test_residual_norm_grad(ctx, rows, width, stream, dtype, pre_norm, post_norm, gate, p):
    bias = "layer" in (pre_norm, post_norm)
    t = case_inputs(rows, width, stream, dtype, pre_norm, post_norm, bias, gate, rows * 37 + width)
    seed, step, scale, eps = 987654321, 3, 0.5, 1e-5
    keep, factor = keep_mask(rows, width, p, seed, step)
    keep = keep.to(DEV)
    d = {k: v.double() if v is not None else None for k, v in t.items()}
    y = d["x"]
    ones = torch.ones(width, dtype=F64, device=DEV)

    def back(v, kind, w, q, q_mag):
        """Gradient, column sums of weight and bias, with magnitudes, of one norm."""
        amp = torch.ones_like(v[:, :1])
        if kind == "layer":
            mean = v.mean(1, keepdim=True)
            v = v - mean
        r = 1.0 / torch.sqrt(v.square().mean(1, keepdim=True) + eps)
        if kind == "layer":
            amp = 1 + (mean.abs() + (v.abs().mean(1, keepdim=True))) * r
        z, u, um = v * r, w * q, w.abs() * q_mag
        dv = r * (u - z * (u * z).mean(1, keepdim=True) - (u.mean(1, keepdim=True) if kind == "layer" else 0.0))
        zm = z.abs() * 1 + (amp - 1)
        dm = r * amp * (um + zm * (um * zm).mean(1, keepdim=True) + (um.mean(1, keepdim=True) if kind == "layer" else 0.0))
        return dv, dm, z, zm, (q * z).sum(0), (q_mag * zm).sum(0), q.sum(0), q_mag.sum(0)

    want, mag = {}, {}
    g, gm = d["dy"], d["dy"].abs()
    if pre_norm:
        dv, dm, _, _, want["dpre"], mag["dpre"], b, bm = back(y, pre_norm, d["pre"], d["dn"], d["dn"].abs())
        if bias:
            want["dpre_bias"], mag["dpre_bias"] = b, bm
        g, gm = g + dv, gm + dm
    want["dx"], mag["dx"] = g, gm
    db, dbm = scale * g, abs(scale) * gm
    db, dbm = torch.where(keep, db * factor, 0.0), torch.where(keep, dbm * factor, 0.0)
    q, qm = (db * d["gate"], dbm * d["gate"].abs()) if gate != "none" else (db, dbm)
    z, zm = d["h"], d["h"].abs()
    if post_norm:
        q, qm, z, zm, want["dpost"], mag["dpost"], b, bm = back(d["h"], post_norm, d["post"], q, qm)
        if bias:
            want["dpost_bias"], mag["dpost_bias"] = b, bm
        z, zm = z * d["post"], zm * d["post"].abs()
        if bias:
            z, zm = z + d["post_bias"], zm + d["post_bias"].abs()
    want["dh"], mag["dh"] = q, qm
    if gate == "vector":
        want["dgate"], mag["dgate"] = (db * z).sum(0), (dbm * zm).sum(0)
    elif gate == "matrix":
        want["dgate"], mag["dgate"] = db * z, dbm * zm
    args = dict(pre_norm=pre_norm, post_norm=post_norm, scale=scale, p=p, seed=seed, step=step, eps=eps, pre=t["pre"], pre_bias=t["pre_bias"], post=t["post"],
                post_bias=t["post_bias"])
    for extra, offset in ((0, 0), (16, 8), (3, 1)):
        v = {k: padded(t[k], extra, offset) if t[k] is not None and t[k].dim() == 2 else t[k] for k in ("x", "h", "gate", "dy", "dn")}
        got = ctx.residual_norm_grad(v["dy"], v["dn"] if pre_norm else None, v["x"], v["h"], gate=v["gate"], **args)
        assert set(got) == set(want)
        for name in want:
            vector = want[name].dim() == 1
            close(got[name], want[name], mag[name], 64 + (rows if vector else 0), F32 if vector else stream if name == "dx" else dtype)
        # over the inputs, the vectors added to what is there
        again = {k: x.clone() for k, x in got.items() if x.dim() == 1}
        res = ctx.residual_norm_grad(v["dy"], v["dn"] if pre_norm else None, v["x"], v["h"], gate=v["gate"], dx=v["dy"], dh=v["h"], accumulate=True, **again, **args)
        for name in got:
            assert torch.equal(res[name], got[name] + got[name] if got[name].dim() == 1 else got[name])


def test_residual_norm_first_block(ctx):
    """Without a block only the norm is taken, and its gradient with what reaches the sum another way."""
    x = torch.randn(100, 96, generator=gen(1)).to(DEV)
    w = torch.randn(96, generator=gen(2)).to(DEV)
    y, n = ctx.residual_norm(x, pre=w, dtype=BF16)
    assert y is x and n.dtype == BF16
    dn, dy = (torch.randn(100, 96, generator=gen(s)).to(DEV) for s in (3, 4))
    got = ctx.residual_norm_grad(dy, dn.to(BF16), x, pre=w)
    assert set(got) == {"dx", "dpre"}
    x64, w64 = x.double().requires_grad_(True), w.double().requires_grad_(True)
    n64 = x64 / torch.sqrt(x64.square().mean(1, keepdim=True) + 1e-6) * w64
    n64.backward(dn.to(BF16).double())
    close(n, n64.detach(), n64.detach().abs(), 64, BF16)
    assert (got["dx"].double() - x64.grad - dy.double()).abs().max() < 64 * U * 16 and (got["dpre"].double() - w64.grad).abs().max() < 164 * U * 200
    only = ctx.residual_norm_grad(None, dn.to(BF16), x, pre=w)
    assert (only["dx"].double() - x64.grad).abs().max() < 64 * U * 16


def test_residual_norm_rows_without_content(ctx):
    """Rows of zeros (padding) give zeros and finite gradients; NaN and infinity stay in their rows."""
    x, h = torch.randn(64, 200, generator=gen(5)).to(DEV), torch.randn(64, 200, generator=gen(6)).to(DEV)
    x[3], h[3] = 0.0, 0.0
    x[7, 5], h[9, 6] = float("nan"), float("inf")
    w = torch.ones(200, device=DEV)
    y, n = ctx.residual_norm(x, h, post_norm="rms", post=w, pre=w, p=0.3, seed=1, step=1)
    assert (y[3] == 0).all() and (n[3] == 0).all()
    clean = torch.tensor([i for i in range(64) if i not in (7, 9)], device=DEV)
    assert y[clean].isfinite().all() and n[clean].isfinite().all() and n[7].isnan().all()
    got = ctx.residual_norm_grad(torch.ones_like(x), torch.ones_like(x), y, h, post_norm="rms", post=w, pre=w, p=0.3, seed=1, step=1)
    assert got["dx"][clean].isfinite().all() and got["dh"][clean].isfinite().all()
    assert ctx.residual_norm(x[:0], h[:0])[1].shape == (0, 200)
    empty = ctx.residual_norm_grad(x[:0], x[:0], x[:0], h[:0], pre=w, post_norm="rms", post=w, gate=w)
    assert (empty["dpre"] == 0).all() and (empty["dpost"] == 0).all() and (empty["dgate"] == 0).all()
    keep = torch.full((200,), 3.0, device=DEV)
    ctx.residual_norm_grad(x[:0], x[:0], x[:0], h[:0], pre=w, dpre=keep, accumulate=True)
    assert (keep == 3.0).all()


@pytest.mark.parametrize("width", [64, 417])
def test_residual_norm_of_rows_too_large_to_square(ctx, width):
    """A row whose squares pass the end of FP32 comes out as zeros, as it does when x is divided by an infinite norm."""
    x = torch.randn(5, width, generator=gen(12)).to(DEV)
    x[2] = 1e25
    x[3, 7] = float("inf")
    _, n = ctx.residual_norm(x)
    want = x.float() / torch.sqrt(x.square().mean(1, keepdim=True) + 1e-6)
    assert (n[2] == 0).all() and (n[3].isnan() == want[3].isnan()).all() and (n[3].nan_to_num(0.0) == 0).all()
    assert (n[[0, 1, 4]] - want[[0, 1, 4]]).abs().max() <= 64 * U * 8


def test_residual_norm_grad_against_differences(ctx):
    """Directional differences of the forward call in FP32: sum(dy y) + sum(dn n) along a random direction of every input."""
    g = gen(11)
    t = {k: torch.randn(40, 72, generator=g).to(DEV) for k in ("x", "h", "gate", "dy", "dn")}
    t.update({k: (1 + 0.2 * torch.randn(72, generator=g)).to(DEV) for k in ("pre", "pre_bias", "post", "post_bias")})
    fixed = dict(pre_norm="layer", post_norm="layer", scale=0.7, p=0.2, seed=4, step=2, eps=1e-5)
    params = ("pre", "pre_bias", "post", "post_bias", "gate")

    def loss(v):
        y, n = ctx.residual_norm(v["x"], v["h"], **{k: v[k] for k in params}, **fixed)
        return (y.double() * t["dy"].double()).sum() + (n.double() * t["dn"].double()).sum()

    y, _ = ctx.residual_norm(t["x"], t["h"], **{k: t[k] for k in params}, **fixed)
    got = ctx.residual_norm_grad(t["dy"], t["dn"], y, t["h"], **{k: t[k] for k in params}, **fixed)
    for name in ("x", "h") + params:
        way = torch.randn(t[name].shape, generator=gen(len(name))).to(DEV)
        step = 2.0 ** -8
        diff = (loss({**t, name: t[name] + step * way}) - loss({**t, name: t[name] - step * way})) / (2 * step)
        slope = (got["d" + name].double() * way.double()).sum()
        # third derivatives are of the size of the first: step^2 of them; the forward values carry 64 u each, 2 * 2880 of them
        scale = got["d" + name].double().norm() * way.double().norm()
        assert (diff - slope).abs() < step ** 2 * 4 * scale + 64 * U * 5760 ** 0.5 * 4 / step, name


def test_residual_norm_repeats_and_replays(pkg):
    """The same bits in every run, on another current stream, and replayed from a graph beside larger eager calls."""
    stream = torch.cuda.Stream()
    c = pkg.Context(0, stream)
    x, h = torch.randn(3000, 256, generator=gen(8)).to(DEV), torch.randn(3000, 256, generator=gen(9)).to(DEV)
    w = torch.ones(256, device=DEV)
    args = dict(pre=w, post_norm="rms", post=w, gate=w, p=0.1, seed=3, step=9)
    y, n = c.residual_norm(x, h, **args)
    first = c.residual_norm_grad(x, h, y, h, **args)
    torch.cuda.synchronize()
    out = {k: torch.empty_like(v) for k, v in first.items()}
    drop = torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        c.residual_norm_grad(x, h, y, h, **args, **out)
        c.dropout(x, 0.5, 1, 2, out=drop)
    big = torch.randn(3000, 2048, device=DEV)
    c.residual_norm_grad(big, big, big, big, pre=torch.ones(2048, device=DEV))   # takes a larger workspace
    for v in out.values():
        v.zero_()
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(out[k], first[k]) for k in first)
    assert torch.equal(drop, c.dropout(x, 0.5, 1, 2))
    del graph
    c.close()


@pytest.mark.parametrize("width", [64, 100, 417, 1000])
def test_residual_norm_wait_that_runs_out(pkg, width):
    """The first row's wait expires (16 bytes more are announced than come): reported once, and the context goes on."""
    c = pkg.Context(0)
    x = torch.randn(300, width, generator=gen(13)).to(DEV)
    w = torch.ones(width, device=DEV)
    y, n = c.residual_norm(x, x, pre=w)
    got = c.residual_norm_grad(x, x, y, x, pre=w)
    c.stats()
    for call in (lambda: c.residual_norm(x, x, pre=w), lambda: c.residual_norm_grad(x, x, y, x, pre=w)):
        c.set_wait_limit(2_000_000, 16)
        call()
        with pytest.raises(pkg.LpError) as e:
            c.stats()
        assert e.value.status == -6
        c.set_wait_limit(2_000_000_000, 0)
        c.stats()
        assert torch.equal(c.residual_norm(x, x, pre=w)[1], n)
        again = c.residual_norm_grad(x, x, y, x, pre=w)
        assert all(torch.equal(again[k], got[k]) for k in got)
    c.close()


def test_block_refusals(pkg, ctx):
    x = torch.zeros(4, 16, device=DEV)
    w = torch.ones(16, device=DEV)
    bad = [lambda: ctx.dropout(x, 1.5, 0, 0), lambda: ctx.dropout(x, float("nan"), 0, 0), lambda: ctx.dropout(x, 0.5, -1, 0), lambda: ctx.dropout(x, 0.5, 0, 1 << 64),
           lambda: ctx.dropout(x, 0.5, 0, 0, row_base=-1), lambda: ctx.dropout(x.half(), 0.5, 0, 0), lambda: ctx.dropout(x.T, 0.5, 0, 0), lambda: ctx.dropout(x.cpu(), 0.5, 0, 0),
           lambda: ctx.dropout(x, 0.5, 0, 0, out=x[:3]), lambda: ctx.dropout(x, 0.5, 0, 0, out=x.bfloat16()),
           lambda: ctx.residual_norm(x, x, eps=0.0), lambda: ctx.residual_norm(x, x, eps=float("inf")), lambda: ctx.residual_norm(x, x, pre_norm="batch"),
           lambda: ctx.residual_norm(x, pre_norm=None), lambda: ctx.residual_norm(x, x, scale=float("nan")), lambda: ctx.residual_norm(x.bfloat16(), x),
           lambda: ctx.residual_norm(x, x[:3]), lambda: ctx.residual_norm(x, x, pre=w[:15]), lambda: ctx.residual_norm(x, x, pre=w.double()), lambda: ctx.residual_norm(x, x, gate=x[:, :8]),
           lambda: ctx.residual_norm(x, x, gate=x.bfloat16()), lambda: ctx.residual_norm(x, x, p=-0.1), lambda: ctx.residual_norm(x, x, pre_norm=None, n=x),
           lambda: ctx.residual_norm(torch.zeros(2, 8193, device=DEV)), lambda: ctx.residual_norm_grad(None, None, None), lambda: ctx.residual_norm_grad(x, None, x, x),
           lambda: ctx.residual_norm_grad(x, x, None, x), lambda: ctx.residual_norm_grad(x, x, x, x, pre=w, accumulate=True), lambda: ctx.residual_norm_grad(x, x, x, x, dpost=w),
           lambda: ctx.residual_norm_grad(x, x, x, x, dh=x[:3]), lambda: ctx.residual_norm_grad(x, x, x, x, pre_norm=None)]
    for i, call in enumerate(bad):
        with pytest.raises(pkg.LpError) as e:
            call()
        assert e.value.status in (-1, -5), i
    assert ctx.dropout(x, 0.5, 0, 0).shape == (4, 16)   # the context is as usable as before
