"""The example model on prepared mini-batches: its scores and every gradient against automatic differentiation of the same model
in 64 bits on the same batch, and training that gets somewhere."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def setup():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2310_00837_amd import helios, sage, workload as W
    sp = W.spec(0)
    g = W.make_graph(sp, 1234, "cpu")
    feats = W.feature_rows(1234, torch.arange(g.n_nodes), sp.dim, sp.dtype)
    h = helios.Helios(0)
    keep = (g.offsets.cuda(), g.indices.cuda(), g.order.to(torch.int32).cuda(), feats[g.order.long()].cuda())
    h.csr_load(keep[0], keep[1])
    h.cache_build(keep[2], g.n_nodes, 0, sp.row_bytes, keep[3], None, None)
    yield sage, W, sp, g, feats, h, sage.Loader(h, sp.batch, sp.fanouts, sp.dim, sp.dtype)
    h.close()


def _mean(x, indptr, col):
    deg = (indptr[1:] - indptr[:-1])
    out = torch.zeros((deg.numel(), x.shape[1]), dtype=x.dtype).index_add(0, torch.repeat_interleave(torch.arange(deg.numel()), deg), x[col.long()])
    return out / deg.clamp_min(1)[:, None]


def _norm(t, g, eps):
    return t / torch.sqrt((t * t).mean(1, keepdim=True) + eps) * g


def _model(sage, b, w):
    x, ip = b.x.double().cpu(), [t.cpu() for t in b.indptr]
    both = torch.cat([torch.cat([x[b.row[k].cpu().long()], _mean(x, ip[k], b.col[k].cpu())], 1) for k in (0, 1)])
    h1 = _norm(torch.relu(both @ w["w1"].t() + w["b1"]), w["g1"], sage.EPS)
    n0 = b.row[0].numel()
    a2 = torch.relu(torch.cat([h1[:n0], _mean(h1, ip[0], b.inner.cpu())], 1) @ w["w2"].t() + w["b2"])
    return _norm(a2 + h1[:n0], w["g2"], sage.EPS) @ w["w3"].t() + w["b3"]


@pytest.mark.parametrize("hidden", [64, 100])
def test_scores_and_gradients(setup, hidden):
    """Single precision: every step is good to some 1e-6 of its largest values and there are about ten of them."""
    sage, W, sp, g, feats, h, loader = setup
    seeds = W.seed_batch(sp, g, 3).cuda()
    b = loader.load(seeds, 77)
    assert torch.equal(b.x[b.row[0].long()].cpu(), feats[seeds.cpu().long()])
    model = sage.Sage(h, sp.dim, hidden, 8, sp.dtype, seed=hidden)
    for k, name in enumerate(("b1", "b2", "b3")):
        model.w[name].copy_(0.1 * torch.randn(model.w[name].shape, generator=torch.Generator().manual_seed(k)))
    w64 = {k: v.double().cpu().requires_grad_(True) for k, v in model.w.items()}
    want = _model(sage, b, w64)
    got, state = model.scores(b)
    assert float((got.double().cpu() - want.detach()).abs().max()) < 1e-5 * float(want.detach().abs().max())
    dscores = torch.randn(want.shape, generator=torch.Generator().manual_seed(9))
    want.backward(dscores.double())
    grads = model.gradients(b, state, dscores.cuda())
    h.sync()
    for name, t in grads.items():
        ref = w64[name].grad
        assert float((t.double().cpu() - ref).abs().max()) < 2e-5 * float(ref.abs().max()), name


def test_training_lowers_the_loss_and_8_bits_serve_it(setup):
    sage, W, sp, g, feats, h, loader = setup
    labels = (feats @ torch.randn((sp.dim, 8), generator=torch.Generator().manual_seed(1))).argmax(1).cuda()
    model = sage.Sage(h, sp.dim, 64, 8, sp.dtype)
    losses = []
    for k in range(60):
        seeds = W.seed_batch(sp, g, k).cuda()
        losses.append(float(model.step(loader.load(seeds, k), labels[seeds.long()], 0.5)))
    assert sum(losses[-10:]) < 0.7 * sum(losses[:10])
    b = loader.load(seeds, 5)
    full, eight = model.scores(b)[0], model.serve(b, model.head_in_8_bits())
    assert float((full.argmax(1) == eight.argmax(1)).float().mean()) > 0.85
    assert float((full - eight).norm() / full.norm()) < 0.1
