"""One attention layer over sampled neighbours, trained and then served, on the rows that
sampling, packing and assembly hand out.

A step takes a group of mini-batches: it samples and packs the group in one call, assembles
each mini-batch's features, adds a learned embedding per node to them, norms the sum, lets
the frontier nodes attend over their sampled neighbours and classifies the seeds.  The
gradients come from the library's own calls; the embeddings' gradient is summed over all
mini-batches of the group, as a sparse list of the nodes that occur.  Serving keeps the
normed rows in 8 bits with a scale per row, looks rows up from there, and lets one node
attend over all of its neighbours.

    python examples/train_attention.py [--steps 30] [--workload T]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2405_05231_amd as dg  # noqa: E402
import synth  # noqa: E402

DEV = "cuda"


class Model:
    """x = features + embedding; y = norm(x); o = attention of y over neighbours; logits of
    (o + y) at the seeds."""

    def __init__(self, nodes: int, dim: int, heads: int, classes: int, seed: int = 0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)

        def rand(*shape, spread):
            return torch.randn(*shape, device=DEV, generator=g) * spread

        self.heads, self.dim = heads, dim
        self.table = rand(nodes, dim, spread=0.1)
        self.weight = torch.ones(dim, device=DEV)
        self.proj = {n: rand(dim, dim, spread=dim ** -0.5) for n in "qkv"}
        self.head = rand(dim, classes, spread=dim ** -0.5)

    def split(self, y):
        return y.view(y.shape[0], self.heads, -1)

    def forward(self, feats, nodes, offsets, indices):
        """feats [n, dim] and nodes [n] of a mini-batch, the lists of its frontier nodes (the
        first rows).  Returns what backward needs."""
        frontier = offsets.numel() - 1
        emb = dg.embed_rows(self.table, nodes)
        norm = dg.norm_rows(emb, self.weight, residual=feats)
        q = self.split(norm.y[:frontier] @ self.proj["q"])
        k, v = self.split(norm.y @ self.proj["k"]), self.split(norm.y @ self.proj["v"])
        att = dg.attend_edges(q, k, v, offsets, indices)
        return dict(norm=norm, q=q, k=k, v=v, att=att, offsets=offsets, indices=indices)

    def logits(self, s, seeds: int):
        return (s["att"].out[:seeds].reshape(seeds, -1) + s["norm"].y[:seeds]) @ self.head

    def backward(self, s, grad_logits):
        """Gradients of a mini-batch: of the projections and the head by name, of the norm's
        weight, and of the embedding rows that it looked up."""
        seeds, frontier = grad_logits.shape[0], s["q"].shape[0]
        y = s["norm"].y
        z = s["att"].out[:seeds].reshape(seeds, -1) + y[:seeds]
        grads = {"head": z.t() @ grad_logits}
        grad_z = grad_logits @ self.head.t()
        grad_o = torch.zeros_like(s["att"].out)
        grad_o[:seeds] = self.split(grad_z)
        g = dg.attend_edges_grad(grad_o, s["q"], s["k"], s["v"], s["att"].out, s["att"].lse,
                                 s["offsets"], s["indices"])
        grad_y = torch.zeros_like(y)
        grad_y[:seeds] += grad_z
        for name, part in (("q", g.q), ("k", g.k), ("v", g.v)):
            part = part.reshape(part.shape[0], -1)
            rows = frontier if name == "q" else y.shape[0]
            grads[name] = y[:rows].t() @ part
            grad_y[:rows] += part @ self.proj[name].t()
        grad_rows, grads["weight"] = dg.norm_rows_grad(grad_y, s["norm"].h, s["norm"].rstd,
                                                       self.weight)
        return grads, grad_rows

    def update(self, grads, nodes, grad_rows, rate):
        for name in "qkv":
            self.proj[name] -= rate * grads[name]
        self.head -= rate * grads["head"]
        self.weight -= rate * grads["weight"]
        rows, sums = dg.embed_rows_grad(grad_rows, nodes, self.table.shape[0], sparse=True)
        self.table.index_add_(0, rows.long(), sums, alpha=-rate)


def batches(w, step: int):
    """A group's mini-batches: node lists, assembled features, and the frontier's lists."""
    dev_slot, feats = w.cache_slot.to(DEV), w.feats.to(DEV)
    sr, pr = dg.sample_pack_group(w.offsets.to(DEV), w.indices.to(DEV), w.seeds.to(DEV),
                                  list(w.cfg.fanouts), w.rng_seed, feats, dev_slot,
                                  batch_base=step * w.cfg.B, direct=True)
    cache = w.cache.to(DEV)
    for b in range(w.cfg.B):
        nodes = sr.batch_nodes(b)
        rows = dg.assemble_batch(cache, pr.chunk(b), pr.loc[b, :nodes.numel()], w.cfg.row_bytes)
        src, dst = sr.batch_edges(b)
        frontier = int(sr.hop_ptr[b, -2])  # the last hop's nodes sample nothing
        yield (nodes.contiguous(), rows.view(torch.float32).view(nodes.numel(), -1),
               dg.edge_offsets(src.contiguous(), frontier), dst.contiguous())


def train(steps: int = 30, workload: str = "T", rate: float = 0.5, log=print):
    """Trains; returns (model, workload, loss of each step)."""
    w = synth.make_workload(workload)
    feats = w.feats.to(DEV)
    dim = feats.shape[1]
    model = Model(w.cfg.n, dim, heads=4, classes=2)
    labels = (feats.sum(1) > 0).long()  # what a model can learn from the features
    seeds, losses = w.seeds.shape[1], []
    for step in range(steps):
        total, grads, all_nodes, all_rows = 0.0, {}, [], []
        for nodes, rows, offsets, indices in batches(w, step):
            s = model.forward(rows, nodes, offsets, indices)
            want = labels[nodes[:seeds].long()]
            logp = torch.log_softmax(model.logits(s, seeds), 1)
            share = 1.0 / (seeds * w.cfg.B)
            total -= float(logp.gather(1, want[:, None]).sum()) * share
            grad_logits = logp.exp()
            grad_logits[torch.arange(seeds, device=DEV), want] -= 1.0
            g, grad_rows = model.backward(s, grad_logits * share)
            for name, x in g.items():
                grads[name] = grads[name] + x if name in grads else x
            all_nodes.append(nodes)
            all_rows.append(grad_rows)
        model.update(grads, torch.cat(all_nodes), torch.cat(all_rows), rate)
        losses.append(total)
        if log and step % 5 == 0:
            log(f"step {step}: loss {total:.4f}")
    return model, w, losses


def serve(model: Model, w, node: int):
    """Logits of one node from rows kept in 8 bits, attending over all of its neighbours."""
    feats = w.feats.to(DEV)
    every = torch.arange(w.cfg.n, dtype=torch.int32, device=DEV)
    kept = dg.norm_rows(dg.embed_rows(model.table, every), model.weight, residual=feats,
                        dtype=torch.float8_e4m3fn)
    offsets, indices = w.offsets.to(DEV), w.indices.to(DEV)
    lo, hi = int(offsets[node]), int(offsets[node + 1])
    listed = torch.cat([every[node:node + 1], indices[lo:hi]])
    y = dg.embed_rows(kept.y, listed, row_scale=kept.scale.view(-1))
    q = model.split(y[:1] @ model.proj["q"])
    k, v = model.split(y @ model.proj["k"]), model.split(y @ model.proj["v"])
    att = dg.attend_edges(q, k, v, torch.tensor([0, hi - lo], device=DEV), every[1:hi - lo + 1])
    return (att.out.reshape(1, -1) + y[:1]) @ model.head


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--steps", type=int, default=30)
    p.add_argument("--workload", default="T")
    a = p.parse_args()
    model, w, losses = train(a.steps, a.workload)
    node = int(w.seeds[0, 0])
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}; served logits of node {node}: "
          f"{serve(model, w, node).flatten().tolist()}")


if __name__ == "__main__":
    main()
