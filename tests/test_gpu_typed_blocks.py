"""Residual blocks over typed nodes: the operators run together as the learned-feature model uses them."""
import numpy as np
import pytest

import workloads as wl

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__ as ge
    ge.build()
    import paper_2506_20818_b200 as p
    return p


def setup(pkg, **kw):
    from paper_2506_20818_b200.learned_features import LearnedFeatures
    g = wl.chung_lu(3000, 12.0, 2.1, seed=0)
    ctx = pkg.Context(0)
    ctx.load_graph(g.n, g.rowptr, g.col, None, wl.node_features(g.n, 8, 0))
    u, v = (torch.from_numpy(x).to("cuda:0") for x in wl.undirected_edge_list(g))
    return ctx, LearnedFeatures(ctx, g.n, width=72, out=64, seed=1, **kw), u, v


def rms(v, w):
    return v / torch.sqrt(v.square().mean(1, keepdim=True) + 1e-6) * w


@pytest.mark.parametrize("types,blocks,dropout", [(1, 1, 0.0), (5, 2, 0.2), (300, 1, 0.5)])
def test_gradients_against_autograd_in_64_bits(pkg, types, blocks, dropout):
    """Every block of the flat gradient within the BF16 path's tolerance (2e-2, relative L2) of autograd on the same loss.  The
    reference takes the path's own ReLU decisions (a unit whose pre-activation lies within the rounding decides either way) and its
    dropout mask, which the dropout operator gives for the same seed, step and rows."""
    ctx, model, u, v = setup(pkg, types=types, blocks=blocks, dropout=dropout)
    src, dst = u[:2000].contiguous(), v[:2000].contiguous()
    _, neg = ctx.sample_negatives(3, 0, 1, src)
    p = {n: model.part(model.params, n).double().clone().requires_grad_(True) for n in model.offset}
    order, ids, offsets, kept, *_ = model.forward_blocks(torch.cat((src, dst, neg)), 0, train=True)
    bounds = offsets.tolist()
    assert bounds[0] == 0 and bounds[-1] == 6000 and len(bounds) == types + 1
    s = p["E"][ids.long()] * model.scale
    n = rms(s, p["pre"][0])
    for i in range(blocks):
        w = p[f"W{i}"].view(types, 72, 72)
        pre = torch.cat([n[lo:hi] @ w[t] + p[f"b{i}"][t] for t, (lo, hi) in enumerate(zip(bounds[:-1], bounds[1:]))])
        h = pre * (kept[i][2] > 0)
        b = rms(h, p["post"][i])
        if dropout > 0:
            b = b * ctx.dropout(torch.ones(6000, 72, device="cuda:0"), dropout, seed=model.seed * blocks + i + 1, step=0).double()
        s = s + p["gate"][i] * b
        n = rms(s, p["pre"][i + 1])
    z = n @ p["W2"] + p["b2"]
    z = torch.empty_like(z).index_copy(0, order, z)
    zs, zd, zn = z.view(3, 2000, -1)
    pos, negs = (zs * zd).sum(1), (zs * zn).sum(1)
    want = (torch.nn.functional.softplus(-pos).sum() + torch.nn.functional.softplus(negs).sum()) / 4000
    want.backward()
    loss = model.step(src, dst, neg)
    assert abs(loss - want.item()) <= 2e-2 * want.item()
    for name in model.offset:
        got, ref = model.part(model.grads, name).double(), p[name].grad
        assert ((got - ref).norm() / ref.norm()).item() <= 2e-2, name
    ctx.stats()
    ctx.close()


def test_training_runs_and_evaluation_drops_nothing(pkg):
    ctx, model, u, v = setup(pkg, types=4, blocks=2, dropout=0.1)
    gen = torch.Generator(device="cuda:0").manual_seed(0)
    for step in range(10):
        pick = torch.randint(0, u.numel(), (4096,), device="cuda:0", generator=gen)
        src, dst = u[pick].contiguous(), v[pick].contiguous()
        _, neg = ctx.sample_negatives(0, step, 1, src)
        assert np.isfinite(model.step(src, dst, neg))
    ids = torch.arange(3000, dtype=torch.int32, device="cuda:0")
    first, again, dropped = (model.forward_blocks(ids, s, train=t)[-1] for s, t in ((0, False), (5, False), (0, True)))
    assert torch.equal(first, again) and not torch.equal(first, dropped) and first.isfinite().all()
    assert torch.isfinite(model.params).all()
    ctx.stats()
    ctx.close()


def test_without_blocks_the_model_is_what_it_was(pkg):
    ctx, model, u, v = setup(pkg)
    assert list(model.offset) == ["E", "W1", "b1", "W2", "b2"] and len(model.matrices) == 2
    ctx.close()
