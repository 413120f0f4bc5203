"""Pins of tests/vector_reference.py: the forms that the GPU tests compare with, against torch's in 64 bits and automatic differentiation."""
import numpy as np
import torch

import vector_reference as vec


def test_lookup_and_its_gradient():
    rng = np.random.default_rng(0)
    table, ids = rng.normal(size=(7, 5)), np.array([3, 0, 6, 3, -1, 7, 3, 2])
    t = torch.from_numpy(table).requires_grad_()
    there = (ids >= 0) & (ids < 7)
    y = torch.zeros(8, 5, dtype=torch.float64)
    y[torch.from_numpy(there)] = torch.nn.functional.embedding(torch.from_numpy(ids[there]), t) * 1.5
    assert np.array_equal(vec.embedding(table, ids, 1.5), y.detach().numpy())
    dy = rng.normal(size=(8, 5))
    (y * torch.from_numpy(dy)).sum().backward()
    grad, size, count = vec.embedding_grad(dy, ids, 7, 1.5)
    assert np.allclose(grad, t.grad.numpy(), rtol=1e-14, atol=0) and list(count) == [1, 0, 1, 3, 0, 0, 1] and (size >= np.abs(grad) - 1e-12).all()


def test_cross_entropy_and_its_gradients():
    rng = np.random.default_rng(1)
    x, w = rng.normal(size=(9, 4)) * 3.0, rng.normal(size=(6, 4))
    labels, share = np.array([0, 5, -1, 2, 6, 3, 3, 1, 0]), rng.random(9)
    tx, tw = (torch.from_numpy(a).requires_grad_() for a in (x, w))
    z = tx @ tw.t()
    counts = (labels >= 0) & (labels < 6)
    each = torch.nn.functional.cross_entropy(z, torch.from_numpy(np.where(counts, labels, -100)), reduction="none", ignore_index=-100)
    loss, lse = vec.cross_entropy(vec.logits(x, w), labels)
    assert np.allclose(loss, each.detach().numpy(), atol=1e-13) and np.allclose(lse, np.where(counts, torch.logsumexp(z, 1).detach().numpy(), 0.0), atol=1e-13)
    (each * torch.from_numpy(share)).sum().backward()
    dx, dw, p, g = vec.cross_entropy_grad(vec.logits(x, w), labels, lse, share, x, w)
    assert np.allclose(dx, tx.grad.numpy(), atol=1e-13) and np.allclose(dw, tw.grad.numpy(), atol=1e-13)
    assert np.allclose(p.sum(1), counts) and (g[~counts] == 0).all()
