"""The lookup of learned vectors, its gradient, and softmax cross entropy with its gradients, in 64 bits from their definitions."""
import numpy as np


def embedding(table, ids, scale):
    there = (ids >= 0) & (ids < len(table))
    y = np.zeros((len(ids), table.shape[1]))
    y[there] = table[ids[there]] * scale
    return y


def embedding_grad(dy, ids, rows, scale):
    """(sums, sums of sizes, entries) of every row of the table."""
    grad, size, count = np.zeros((rows, dy.shape[1])), np.zeros((rows, dy.shape[1])), np.zeros(rows, dtype=np.int64)
    there = (ids >= 0) & (ids < rows)
    np.add.at(grad, ids[there], dy[there] * scale)
    np.add.at(size, ids[there], np.abs(dy[there] * scale))
    np.add.at(count, ids[there], 1)
    return grad, size, count


def logits(x, weight):
    return x @ weight.T


def cross_entropy(z, labels):
    """(loss, log-sum) of every row."""
    counts = (labels >= 0) & (labels < z.shape[1])
    top = z.max(1)
    lse = top + np.log(np.exp(z - top[:, None]).sum(1))
    at = np.where(counts, labels, 0)
    return np.where(counts, lse - z[np.arange(len(z)), at], 0.0), np.where(counts, lse, 0.0)


def cross_entropy_grad(z, labels, lse, share, x, weight):
    """(dx, dweight, p, g): p the softmax by the given lse (0 where a row does not count), g = share (p - one-hot)."""
    counts = (labels >= 0) & (labels < z.shape[1])
    p = np.where(counts[:, None], np.exp(np.where(counts[:, None], z - lse[:, None], 0.0)), 0.0)
    g = p.copy()
    g[np.flatnonzero(counts), labels[counts]] -= 1.0
    g *= np.where(counts, share, 0.0)[:, None]
    return g @ weight, g.T @ x, p, g
