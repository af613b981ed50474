"""The training example: its gradients against autograd on a plain model, its training, and
its serving path in 8 bits against the plain model in 32."""
import os
import sys

import pytest
import torch

from conftest import ROOT

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import train_attention
    return train_attention


def plain_logits(model, feats, nodes, offsets, indices, seeds, table, weight, proj, head):
    """The model's formulas in 64 bits, for autograd."""
    x = table[nodes.long()] + feats.double()
    y = x * (x.square().mean(1, keepdim=True) + 1e-6).rsqrt() * weight
    n, frontier, H = y.shape[0], offsets.numel() - 1, model.heads
    q = (y[:frontier] @ proj["q"]).view(frontier, H, -1)
    k, v = (y @ proj["k"]).view(n, H, -1), (y @ proj["v"]).view(n, H, -1)
    row = torch.repeat_interleave(torch.arange(frontier, device=DEV), offsets.diff())
    at = indices.long()
    s = (q[row] * k[at]).sum(2) * q.shape[2] ** -0.5
    p = torch.zeros(frontier, H, dtype=torch.float64, device=DEV).index_add(0, row, s.exp())
    p = s.exp() / p[row]
    o = torch.zeros_like(q).index_add(0, row, p[:, :, None] * v[at])
    return (o[:seeds].reshape(seeds, -1) + y[:seeds]) @ head


def test_gradients_against_autograd(ex):
    import synth
    w = synth.make_workload("T")
    dim = w.feats.shape[1]
    model = ex.Model(w.cfg.n, dim, heads=4, classes=2, seed=3)
    seeds = w.seeds.shape[1]
    nodes, rows, offsets, indices = next(iter(ex.batches(w, 0)))
    s = model.forward(rows, nodes, offsets, indices)
    leaf = lambda x: x.double().requires_grad_()  # noqa: E731
    table, weight, head = leaf(model.table), leaf(model.weight), leaf(model.head)
    proj = {n: leaf(p) for n, p in model.proj.items()}
    want = plain_logits(model, rows, nodes, offsets, indices, seeds, table, weight, proj, head)
    got = model.logits(s, seeds)
    # 32-bit products over 16 to 64 terms of magnitudes below 10: 1e-4 is several times their
    # bound, and of a gradient's largest value
    assert (got - want).abs().max() <= 1e-4
    g_logits = torch.randn(seeds, 2, device=DEV)
    want.backward(g_logits.double())
    grads, grad_rows = model.backward(s, g_logits)
    import paper_2405_05231_amd as dg
    grad_table = dg.embed_rows_grad(grad_rows, nodes, w.cfg.n)
    for x, y in ((grad_table, table.grad), (grads["weight"], weight.grad),
                 (grads["head"], head.grad), *((grads[n], proj[n].grad) for n in "qkv")):
        assert (x - y).abs().max() <= 1e-4 * float(y.abs().max())


def test_training_lowers_the_loss_and_serving_follows_the_model(ex):
    import synth  # noqa: F401
    model, w, losses = ex.train(steps=12, log=None)
    assert losses[-1] < 0.7 * losses[0]
    node = int(w.seeds[0, 0])
    got = ex.serve(model, w, node)
    lo, hi = int(w.offsets[node]), int(w.offsets[node + 1])
    listed = torch.cat([torch.tensor([node], dtype=torch.int32), w.indices[lo:hi]]).to(DEV)
    want = plain_logits(model, w.feats.to(DEV)[listed.long()], listed,
                        torch.tensor([0, hi - lo], device=DEV),
                        torch.arange(1, hi - lo + 1, dtype=torch.int32, device=DEV), 1,
                        model.table.double(), model.weight.double(),
                        {n: p.double() for n, p in model.proj.items()}, model.head.double())
    # rows are off by up to 2^-4 of their values in 8 bits
    assert (got - want).abs().max() <= 0.15 * float(want.abs().max()) + 0.15
