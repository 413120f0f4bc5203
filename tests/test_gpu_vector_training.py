"""One training step of a model that learns a vector for every node, through the library's operators in a row: lookup, layer norm, cross entropy over all nodes with the
table as weight (so its gradient comes from both ends), and the clipped gradients; against the same step in 64 bits by automatic differentiation."""
import numpy as np
import pytest
import torch

from test_gpu_training_ops import DEV, ctx, f64, _name_the_case  # noqa: F401  (fixtures among them)

pytestmark = pytest.mark.gpu
EPS, MAX_NORM, SCALE = 1e-5, 0.05, 4.0


class Step:
    """Buffers of a step, and the step."""

    def __init__(self, ctx, n, nodes, dim):  # noqa: F811
        from paper_2505_10806_amd import binding as B
        empty = lambda *shape: torch.zeros(*shape, device=DEV)                                            # noqa: E731
        self.ctx, self.n, self.nodes, self.dim = ctx, n, nodes, dim
        self.v, self.h, self.dh, self.dv = (empty(n, dim) for _ in range(4))
        self.mean, self.rstd, self.loss, self.lse, self.norm = empty(n), empty(n), empty(n), empty(n), empty(1)
        self.grads = dict(table=empty(nodes, dim), gamma=empty(dim), beta=empty(dim))
        self.list = B.TensorList(list(self.grads.values()))

    def __call__(self, table, gamma, beta, ids, labels, n_dev, stream=None):
        c, n, dim, g = self.ctx, self.n, self.dim, self.grads
        c.embedding(table, self.nodes, ids, n, dim, self.v, scale=SCALE, n_dev=n_dev, stream=stream)
        c.layer_norm(self.v, n, dim, gamma, beta, EPS, self.h, self.mean, self.rstd, n_dev=n_dev, stream=stream)
        c.cross_entropy(self.h, n, dim, table, self.nodes, labels, self.loss, self.lse, n_dev=n_dev, stream=stream)
        c.cross_entropy_grad(self.h, n, dim, table, self.nodes, labels, self.lse, self.dh, g["table"], scale=1.0 / n, n_dev=n_dev, stream=stream)
        c.layer_norm_grad(self.dh, self.v, n, dim, gamma, self.mean, self.rstd, self.dv, g["gamma"], g["beta"], n_dev=n_dev, stream=stream)
        c.embedding_grad(self.dv, ids, n, dim, self.nodes, g["table"], scale=SCALE, add=True, n_dev=n_dev, stream=stream)
        c.clip_grad_norm(self.list, MAX_NORM, self.norm, stream=stream)


def by_autograd(table, gamma, beta, ids, labels, n):
    """Losses, norm and clipped gradients of the step in 64 bits (rows without a label do not count; ids outside the table read zeros)."""
    t, ga, be = (torch.from_numpy(a).requires_grad_() for a in (table, gamma, beta))
    there = torch.from_numpy((ids >= 0) & (ids < len(table)))
    v = torch.where(there[:, None], t[torch.from_numpy(np.where(there, ids, 0))] * SCALE, torch.zeros((), dtype=torch.float64))
    m = v.mean(1, keepdim=True)
    h = (v - m) / torch.sqrt(((v - m) ** 2).mean(1, keepdim=True) + EPS) * ga + be
    z = h @ t.t()
    counts = torch.from_numpy((labels >= 0) & (labels < len(table)))
    picked = z.gather(1, torch.from_numpy(np.where(counts, labels, 0))[:, None])[:, 0]
    loss = torch.where(counts, torch.logsumexp(z, 1) - picked, torch.zeros((), dtype=torch.float64))
    (loss.sum() / n).backward()
    grads = [x.grad for x in (t, ga, be)]
    norm = float(torch.sqrt(sum((g ** 2).sum() for g in grads)))
    return loss.detach().numpy(), norm, [(g * min(1.0, MAX_NORM / norm)).numpy() for g in grads]


def inputs(rng, n, nodes, dim):
    table = (rng.normal(size=(nodes, dim)) * dim ** -0.5).astype(np.float32)
    gamma, beta = (1.0 + 0.1 * rng.normal(size=dim)).astype(np.float32), (0.1 * rng.normal(size=dim)).astype(np.float32)
    ids = np.where(rng.random(n) < 0.05, -1, rng.integers(0, nodes, n))
    labels = np.where(rng.random(n) < 0.1, -1, rng.integers(0, nodes, n))
    return table, gamma, beta, ids, labels


def on_gpu(arrays):
    return [torch.from_numpy(a.astype(np.int32) if a.dtype == np.int64 else a).to(DEV) for a in arrays]


def compare(step, want, n, live):
    """Every sum has at most `nodes` + `dim` terms of 32 bits, whose errors pass through four operators: 2^-24 sqrt(terms) each, of the largest number around."""
    loss, norm, grads = want
    bound = 2.0 ** -24 * 64.0 * np.sqrt(step.nodes + step.dim)
    assert np.abs(f64(step.loss)[:live] - loss[:live]).max() <= bound * max(1.0, np.abs(loss).max())
    assert abs(float(step.norm) - norm) <= bound * norm
    for got, g in zip(step.grads.values(), grads):
        assert np.abs(f64(got) - g).max() <= bound * np.abs(g).max()


@pytest.mark.parametrize("n,nodes,dim", [(300, 1000, 64), (64, 5000, 100), (200, 47, 130)])
def test_step_is_that_of_automatic_differentiation(ctx, n, nodes, dim):  # noqa: F811
    rng = np.random.default_rng(n)
    arrays = inputs(rng, n, nodes, dim)
    step = Step(ctx, n, nodes, dim)
    step(*on_gpu(arrays), None)
    compare(step, by_autograd(*[a.astype(np.float64) if a.dtype == np.float32 else a for a in arrays], n), n, n)


def test_step_recorded_and_replayed_on_batches_of_other_lengths(ctx):  # noqa: F811
    """The counts stay on the device: one recording serves batches of every length up to its own."""
    rng = np.random.default_rng(5)
    n, nodes, dim = 256, 900, 64
    side, n_dev = torch.cuda.Stream(), torch.zeros(1, dtype=torch.int32, device=DEV)
    place = on_gpu(inputs(rng, n, nodes, dim))
    step = Step(ctx, n, nodes, dim)
    with torch.cuda.stream(side):
        step(*place, n_dev, stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(*place, n_dev, stream=torch.cuda.current_stream())
    for live in (256, 31, 1, 200):
        arrays = list(inputs(rng, n, nodes, dim))
        for to, a in zip(place, on_gpu(arrays)):
            to.copy_(a)
        n_dev.fill_(live)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        arrays[3], arrays[4] = arrays[3][:live], arrays[4][:live]
        compare(step, by_autograd(*[a.astype(np.float64) if a.dtype == np.float32 else a for a in arrays], n), n, live)
