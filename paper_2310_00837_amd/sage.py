"""A small GraphSAGE model on prepared mini-batches: training step by step, and serving in 8 bits.

It runs the library's path from the seeds to the model's gradients: helios_prepare_batch and helios_make_blocks, then
per layer the neighbour mean, the product with bias and activation and the norm with its residual, and their gradients
back to the weights.  Two hops, two layers and a head (Sec. 4.1: 2-hop GraphSAGE):

    h1 = norm(relu([x | mean x] W1^T + b1))                  for the seeds and the first hop's nodes
    h2 = norm(relu([h1 | mean h1] W2^T + b2) + h1)           for the seeds
    scores = h2 W3^T + b3

Usage: python -m paper_2310_00837_amd.sage [steps]     (synthetic graph, features and labels; needs a GPU)
"""
from __future__ import annotations

import sys
from dataclasses import dataclass
from typing import Dict, List

import torch

from paper_2310_00837_amd import helios
from paper_2310_00837_amd import workload as W

EPS = 1e-6


@dataclass
class Batch:
    """A prepared two-hop mini-batch, cut to its size: feature rows and the hops in local numbering."""
    x: torch.Tensor                 # [unique nodes, features]
    indptr: List[torch.Tensor]      # int64[n_h + 1] per hop
    row: List[torch.Tensor]         # int32[n_h]: rows of x of the hop's nodes
    col: List[torch.Tensor]         # int32: rows of x of their samples
    inner: torch.Tensor             # int32: for the seeds' samples, the row of [seeds; first hop's nodes] that holds them


class Loader:
    """Prepares batches of one size on a context whose graph and cache are loaded."""

    def __init__(self, h: helios.Helios, n_seeds: int, fanouts, dim: int, dtype: torch.dtype):
        assert len(fanouts) == 2
        dev = h.device
        self.h, self.fanouts, self.dim, self.dtype = h, list(fanouts), dim, dtype
        self.hops = helios.alloc_hops(n_seeds, fanouts, dev)
        cap = n_seeds + sum(hb.flat.numel() for hb in self.hops)
        ints = lambda n: torch.empty(n, dtype=torch.int32, device=dev)  # noqa: E731
        pinned = lambda n: torch.zeros(n, dtype=torch.int64).pin_memory()  # noqa: E731
        self.sizes, self.n_unique, self.stats = pinned(4), pinned(1), pinned(4)
        self.unique, self.miss = ints(cap), [ints(cap) for _ in range(3)]
        self.out = torch.empty((cap, dim), dtype=dtype, device=dev)
        self.row = [ints(hb.frontier.numel()) for hb in self.hops]
        self.col = [ints(hb.flat.numel()) for hb in self.hops]
        h.reserve(cap)

    def load(self, seeds: torch.Tensor, rng_seed: int) -> Batch:
        h = self.h
        h.prepare_batch(seeds, self.fanouts, rng_seed, self.hops, self.sizes, self.unique, None, self.n_unique, self.out, *self.miss, self.stats)
        h.make_blocks(self.hops, self.row, self.col)
        h.gather_miss(self.miss[0], self.miss[2], self.miss[0].numel(), self.stats[3:4], self.out)
        h.sync()
        u, (n0, e0, n1, e1) = int(self.n_unique), self.sizes.tolist()
        row, col = [self.row[0][:n0], self.row[1][:n1]], [self.col[0][:e0], self.col[1][:e1]]
        where = torch.empty(u, dtype=torch.int32, device=h.device)       # row of x -> place among the first hop's nodes
        where[row[1].long()] = torch.arange(n1, dtype=torch.int32, device=h.device)
        return Batch(self.out[:u], [self.hops[0].indptr[:n0 + 1], self.hops[1].indptr[:n1 + 1]], row, col, where[col[0].long()] + n0)


class Sage:
    """Weights, and the calls of a training step in their order.  Works on the context's stream (torch's current one)."""

    def __init__(self, h: helios.Helios, dim: int, hidden: int, classes: int, dtype: torch.dtype, seed: int = 0):
        self.h, self.hidden, self.dtype = h, hidden, dtype
        gen = torch.Generator().manual_seed(seed)
        new = lambda m, k: (torch.randn((m, k), generator=gen) * k ** -0.5).to(dtype).to(h.device)  # noqa: E731
        self.w: Dict[str, torch.Tensor] = {"w1": new(hidden, 2 * dim), "w2": new(hidden, 2 * hidden), "w3": new(classes, hidden)}
        for name, n in (("b1", hidden), ("b2", hidden), ("b3", classes)):
            self.w[name] = torch.zeros(n, dtype=dtype, device=h.device)
        for name in ("g1", "g2"):
            self.w[name] = torch.ones(hidden, dtype=dtype, device=h.device)

    def _new(self, *shape, dtype=None):
        return torch.empty(shape, dtype=dtype or self.dtype, device=self.h.device)

    def _features(self, b: Batch):
        """The last hidden rows of the seeds in front of their norm, and what the backward pass needs."""
        h, w, d, m = self.h, self.w, b.x.shape[1], self.hidden
        n0, n1 = b.row[0].numel(), b.row[1].numel()
        s = {"both1": self._new(n0 + n1, 2 * d), "both2": self._new(n0, 2 * m)}
        for hop, rows in ((0, s["both1"][:n0]), (1, s["both1"][n0:])):
            h.block_mean(b.x, b.indptr[hop], b.col[hop], rows[:, d:], row=b.row[hop], own=rows[:, :d])
        s["z1"], s["a1"], s["h1"] = (self._new(n0 + n1, m) for _ in range(3))
        h.linear(s["both1"], w["w1"], s["a1"], bias=w["b1"], act=helios.ACT_RELU, pre=s["z1"])
        h.rms_norm(s["a1"], s["h1"], EPS, gain=w["g1"])
        h.block_mean(s["h1"], b.indptr[0], b.inner, s["both2"][:, m:], own=s["both2"][:, :m])
        s["z2"], s["a2"] = self._new(n0, m), self._new(n0, m)
        h.linear(s["both2"], w["w2"], s["a2"], bias=w["b2"], act=helios.ACT_RELU, pre=s["z2"])
        return s

    def scores(self, b: Batch):
        """(class scores in single precision, state for gradients())"""
        h, w, s = self.h, self.w, self._features(b)
        n0 = b.row[0].numel()
        s["t2"], s["h2"] = self._new(n0, self.hidden), self._new(n0, self.hidden)
        h.rms_norm(s["a2"], s["h2"], EPS, gain=w["g2"], residual=s["h1"][:n0], total=s["t2"])
        out = self._new(n0, w["w3"].shape[0], dtype=torch.float32)
        h.linear(s["h2"], w["w3"], out, bias=w["b3"].float())
        return out, s

    def gradients(self, b: Batch, s, dscores: torch.Tensor) -> Dict[str, torch.Tensor]:
        h, w, m = self.h, self.w, self.hidden
        n0, n = b.row[0].numel(), s["h1"].shape[0]
        g = {name: torch.empty_like(t) for name, t in w.items()}
        db3 = torch.empty(g["b3"].shape, dtype=torch.float32, device=h.device)
        dh2, dt2, dboth2, dh1, da1 = self._new(n0, m), self._new(n0, m), self._new(n0, 2 * m), self._new(n, m), self._new(n, m)
        h.linear_grad(s["h2"], w["w3"], dscores, dx=dh2, dw=g["w3"], dbias=db3)
        g["b3"].copy_(db3)
        h.rms_norm_grad(s["t2"], dh2, dt2, EPS, gain=w["g2"], dgain=g["g2"])
        h.linear_grad(s["both2"], w["w2"], dt2, act=helios.ACT_RELU, pre=s["z2"], dx=dboth2, dw=g["w2"], dbias=g["b2"])
        dboth2[:, :m] += dt2                                     # h1 is also the residual
        own = torch.arange(n0, dtype=torch.int32, device=h.device)
        src_indptr, src_entry = self._new(n + 1, dtype=torch.int32), self._new(b.inner.numel() + n0, dtype=torch.int32)
        h.block_transpose(b.indptr[0], b.inner, n, src_indptr, src_entry, row=own)
        h.block_mean_grad(b.indptr[0], src_indptr, src_entry, dboth2[:, m:], dh1, down=dboth2[:, :m])
        h.rms_norm_grad(s["a1"], dh1, da1, EPS, gain=w["g1"], dgain=g["g1"])
        h.linear_grad(s["both1"], w["w1"], da1, act=helios.ACT_RELU, pre=s["z1"], dw=g["w1"], dbias=g["b1"])
        return g

    def step(self, b: Batch, labels: torch.Tensor, rate: float) -> torch.Tensor:
        """One step of gradient descent on the mean cross-entropy; returns the loss (on the GPU)."""
        scores, s = self.scores(b)
        logp = torch.log_softmax(scores, 1)
        n = labels.numel()
        dscores = torch.exp(logp)
        dscores[torch.arange(n, device=labels.device), labels] -= 1.0
        g = self.gradients(b, s, dscores / n)
        for name, t in self.w.items():
            t.sub_(rate * g[name])
        return -logp[torch.arange(n, device=labels.device), labels].mean()

    def head_in_8_bits(self):
        """The head's weights as serve() takes them: laid out once."""
        q, scale = self._new(*self.w["w3"].shape, dtype=torch.float8_e4m3fn), self._new(self.w["w3"].shape[0], dtype=torch.float32)
        self.h.quantize_rows(self.w["w3"], q, scale)
        return q, scale, self.w["b3"].float()

    def serve(self, b: Batch, head) -> torch.Tensor:
        """Class scores with the last norm and the head's product in 8 bits."""
        h, s, n0 = self.h, self._features(b), b.row[0].numel()
        h8, scale = self._new(n0, self.hidden, dtype=torch.float8_e4m3fn), self._new(n0, dtype=torch.float32)
        h.rms_norm(s["a2"], h8, EPS, gain=self.w["g2"], residual=s["h1"][:n0], y_scale=scale)
        out = self._new(n0, head[0].shape[0], dtype=torch.float32)
        h.linear(h8, head[0], out, bias=head[2], x_scale=scale, w_scale=head[1])
        return out


def main(steps: int = 40) -> None:
    sp = W.spec(0)
    g = W.make_graph(sp, 1234, "cpu")
    feats = W.feature_rows(1234, torch.arange(g.n_nodes), sp.dim, sp.dtype)
    classes = 8
    labels = (feats @ torch.randn((sp.dim, classes), generator=torch.Generator().manual_seed(1))).argmax(1).cuda()
    h = helios.Helios(0)
    offsets, indices, order = g.offsets.cuda(), g.indices.cuda(), g.order.to(torch.int32).cuda()
    h.csr_load(offsets, indices)
    table = feats[g.order.long()].cuda()                         # every row in HBM, in rank order
    h.cache_build(order, g.n_nodes, 0, sp.row_bytes, table, None, None)
    loader = Loader(h, sp.batch, sp.fanouts, sp.dim, sp.dtype)
    model = Sage(h, sp.dim, 128, classes, sp.dtype)
    for k in range(steps):
        seeds = W.seed_batch(sp, g, k).cuda()
        loss = model.step(loader.load(seeds, W.batch_rng_seed(1234, k)), labels[seeds.long()], 0.5)
        if k % 10 == 0 or k == steps - 1:
            print(f"step {k}: loss {float(loss):.4f}", flush=True)
    b = loader.load(seeds, 1)
    full, eight = model.scores(b)[0], model.serve(b, model.head_in_8_bits())
    print(f"classes that the scores in 8 bits agree on: {float((full.argmax(1) == eight.argmax(1)).float().mean()):.3f}")
    h.close()


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 40)
