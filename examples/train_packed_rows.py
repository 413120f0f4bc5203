"""Trains a one-layer GraphSAGE classifier on feature rows of 4-bit numbers, from the schedule to the clipped update.

    python examples/train_packed_rows.py [--workload tiny] [--steps 60]

The feature stores are packed once (the remote one where it lies, in pinned memory): a row of 64 floats, 256 bytes, becomes 36.  From
there the data path moves packed rows: the cache holds them, the gather assembles a batch's.  A step projects the seeds' own rows and the
means of their sampled neighbours' with packed weights, normalises the sum and classifies it; its gradients go back through
layer norm and the two products to the 32-bit weights, clipped by their norm together.  Everything but the classifier's small dense layer runs in
the library's kernels.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import synth
from paper_2505_10806_amd import binding as B

EPS = 1e-5


class Model:
    """y = relu(layer_norm(x_v W_self^T + mean(x_u) W_mean^T)) W_out^T; 32-bit weights, packed anew before each step's products."""

    def __init__(self, dim, hidden, classes, batch, device, seed):
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        normal = lambda *shape: torch.randn(*shape, generator=gen, device=device) * shape[-1] ** -0.5     # noqa: E731
        self.dim, self.hidden = dim, hidden
        self.weights = dict(own=normal(hidden, dim), mean=normal(hidden, dim), out=normal(classes, hidden),
                            gamma=torch.ones(hidden, device=device), beta=torch.zeros(hidden, device=device))
        self.grads = {k: torch.zeros_like(w) for k, w in self.weights.items()}
        self.velocity = {k: torch.zeros_like(w) for k, w in self.weights.items()}
        self.packed = {k: B.mx4_rows(hidden, dim, device) for k in ("own", "mean")}
        empty = lambda *shape: torch.empty(*shape, device=device)                                         # noqa: E731
        self.z, self.z_mean, self.h, self.dz = (empty(batch, hidden) for _ in range(4))
        self.mean, self.rstd, self.norm = empty(batch), empty(batch), empty(1)
        self.list = B.TensorList(list(self.grads.values()))      # clipped where they are

    def step(self, ctx, own_rows, mean_rows, n, labels, rate, max_norm):
        """One update from the packed rows of n seeds and of their neighbours' means; returns the loss (a device scalar)."""
        w, g, dim, hidden = self.weights, self.grads, self.dim, self.hidden
        for k, packed in self.packed.items():
            ctx.mx4_quantize(w[k], hidden, dim, packed)
        ctx.mx4_matmul(own_rows, n, self.packed["own"], hidden, dim, self.z)
        ctx.mx4_matmul(mean_rows, n, self.packed["mean"], hidden, dim, self.z_mean)
        z = self.z[:n].add_(self.z_mean[:n])
        ctx.layer_norm(z, n, hidden, w["gamma"], w["beta"], EPS, self.h, self.mean, self.rstd)

        hot = torch.relu(self.h[:n])
        log_p = torch.log_softmax(hot @ w["out"].t(), 1)
        loss = -log_p.gather(1, labels[:, None]).mean()
        d_logits = log_p.exp()
        d_logits.scatter_add_(1, labels[:, None], torch.full((n, 1), -1.0, device=d_logits.device))
        d_logits /= n
        torch.mm(d_logits.t(), hot, out=g["out"])
        d_h = (d_logits @ w["out"]) * (self.h[:n] > 0)

        ctx.layer_norm_grad(d_h, z, n, hidden, w["gamma"], self.mean, self.rstd, self.dz, g["gamma"], g["beta"])
        ctx.mx4_matmul_grad(self.dz, own_rows, n, hidden, dim, g["own"])
        ctx.mx4_matmul_grad(self.dz, mean_rows, n, hidden, dim, g["mean"])
        ctx.clip_grad_norm(self.list, max_norm, self.norm)
        for k in w:
            self.velocity[k].mul_(0.9).add_(g[k])
            w[k].sub_(self.velocity[k], alpha=rate)
        return loss


def train(workload="tiny", steps=60, hidden=128, classes=8, fanout=10, rate=0.1, max_norm=1.0, seed=2025, device="cuda:0"):
    """Returns the losses and the gradients' norms, one of each per step."""
    wl = synth.build_workload(workload, seed=seed, device=device)
    cfg, dim = wl.cfg, wl.cfg.feat_dim
    ctx = B.Context(torch.device(device).index or 0)

    # the stores, packed: what the cache and the gather see is rows of `words` floats
    words = B.mx4_row_words(dim)
    local, remote = B.mx4_rows(wl.n_local, dim, device), B.mx4_rows(wl.n_remote, dim, "cpu", pin_memory=True)
    ctx.mx4_quantize(wl.local_store, wl.n_local, dim, local)
    ctx.mx4_quantize(wl.remote_store, wl.n_remote, dim, remote)

    # labels that the features decide: the largest of a few directions of a node's own row
    gen = torch.Generator(device=device)
    gen.manual_seed(seed + 1)
    labels = (wl.features @ torch.randn(dim, classes, generator=gen, device=device)).argmax(1)

    # a cache of packed rows: for the bytes of the workload's cache seven times as many of them
    csr = B.CsrGraph(wl.row_ptr, wl.col_idx)
    batch, fanouts = cfg.batch_size, (fanout,)
    bufs = B.BlockBuffers(cfg.num_nodes, wl.nnz, batch, fanouts, device)
    most = bufs.frontier_ub[1]
    capacity = min(wl.n_remote, wl.capacity_rows * 4 * dim // (4 * words))
    cache = B.FeatureCache(cfg.num_nodes, capacity, local.shape[1], device)
    counts = torch.zeros(cfg.num_nodes, dtype=torch.int32, device=device)
    order = ctx.epoch_schedule(wl.train_ids, wl.seed, 0)
    ctx.access_histogram(order, order.numel(), counts)
    ctx.build_cache(counts, wl.home, remote, words, cache)

    rows, mean_rows = B.mx4_rows(most, dim, device), B.mx4_rows(batch, dim, device)
    numbers, means = torch.empty(most, wl.stride, device=device), torch.empty(batch, wl.stride, device=device)
    stats = torch.zeros(3, dtype=torch.int64, device=device)
    side = torch.cuda.Stream(device)
    model = Model(dim, hidden, classes, batch, device, seed)
    losses, norms = [], []
    for step in range(steps):
        at = step * batch % max(order.numel() - batch + 1, 1)
        seeds = order[at:at + batch]
        n, n_nodes = seeds.numel(), bufs.tier_off[2:]
        ctx.sample_blocks(csr, seeds, n, fanouts, wl.seed, step, bufs)
        ctx.gather_features(bufs.nodes, most, cache, local, remote, words, rows, stats, n_dev=n_nodes, miss_stream=side)
        ctx.mx4_dequantize(rows, most, dim, numbers, n_dev=n_nodes)
        ctx.mean_aggregate(bufs.indptr[0], bufs.nbr_local[0], n, numbers, dim, means)
        ctx.mx4_quantize(means, n, dim, mean_rows)
        losses.append(model.step(ctx, rows, mean_rows, n, labels[seeds.long()], rate, max_norm))
        norms.append(model.norm.clone())
    torch.cuda.synchronize()
    ctx.close()
    return [float(x) for x in losses], [float(x) for x in norms]


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--workload", default="tiny")
    p.add_argument("--steps", type=int, default=60)
    a = p.parse_args()
    losses, norms = train(a.workload, a.steps)
    for i in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {i:4d}  loss {losses[i]:.4f}  norm of the gradients {norms[i]:.3f}")
    print(f"last       loss {losses[-1]:.4f}")


if __name__ == "__main__":
    main()
