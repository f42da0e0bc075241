"""The example that runs the operators together: learned node features trained with orthogonalised updates."""
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


def setup(pkg):
    from paper_2506_20818_b200.learned_features import LearnedFeatures
    g = wl.chung_lu(3000, 12.0, 2.1, seed=0)
    ctx = pkg.Context(0)
    ctx.load_graph(g.n, g.rowptr, g.col, None, wl.node_features(g.n, 8, 0))
    u, v = (torch.from_numpy(x).to("cuda:0") for x in wl.undirected_edge_list(g))
    return ctx, LearnedFeatures(ctx, g.n, width=64, hidden=128, out=64, seed=1), u, v


def test_gradients_against_autograd_in_64_bits(pkg):
    """Every block of the flat gradient within the BF16 path's tolerance (2e-2, relative L2) of autograd on the same loss.  A hidden
    unit whose pre-activation lies within the rounding of the BF16 path decides its ReLU either way; there, and only there, the
    reference takes the path's decision (one unit in a thousand decided otherwise is 3 % of a gradient)."""
    ctx, model, u, v = setup(pkg)
    src, dst = u[:2000].contiguous(), v[:2000].contiguous()
    _, neg = ctx.sample_negatives(3, 0, 1, src)
    p = {n: model.part(model.params, n).double().clone().requires_grad_(True) for n in model.offset}
    ids = torch.cat((src, dst, neg)).long()
    x = p["E"][ids] * model.scale
    pre = x @ p["W1"] + p["b1"]
    mine = model.forward(ids.int())[1] > 0
    with torch.no_grad():  # x and W1 are rounded to BF16 (2^-9 each, relative), the accumulator adds 2^-22 per term
        window = 2.0**-8 * (x.abs() @ p["W1"].abs())
    assert ((pre > 0) == mine)[pre.abs() > window].all()
    z = (pre * mine) @ p["W2"] + p["b2"]
    zs, zd, zn = z.view(3, 2000, -1)
    pos, negs = (zs * zd).sum(1), (zs * zn).sum(1)
    want = (torch.nn.functional.softplus(-pos).sum() + torch.nn.functional.softplus(negs).sum()) / 4000
    want.backward()
    loss = model.step(src, dst, neg)
    assert abs(loss - want.item()) <= 2e-2 * want.item()
    for n in model.offset:
        got, ref = model.part(model.grads, n).double(), p[n].grad
        assert ((got - ref).norm() / ref.norm()).item() <= 2e-2, n
    ctx.close()


def test_training_lowers_the_loss(pkg):
    ctx, model, u, v = setup(pkg)
    gen = torch.Generator(device="cuda:0").manual_seed(0)
    losses = []
    for step in range(60):
        pick = torch.randint(0, u.numel(), (4096,), device="cuda:0", generator=gen)
        src, dst = u[pick].contiguous(), v[pick].contiguous()
        _, neg = ctx.sample_negatives(0, step, 1, src)
        losses.append(model.step(src, dst, neg))
    assert all(np.isfinite(losses))
    assert np.mean(losses[-5:]) < 0.8 * np.mean(losses[:5])
    ctx.stats()
    ctx.close()
