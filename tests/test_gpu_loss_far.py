"""Softmax cross entropy and its gradients on an MI355X where a row or a class stands far from the others."""
import numpy as np
import pytest
import torch

import training_reference as ref
from test_gpu_loss_ops import inputs, on_gpu
from test_gpu_training_ops import DEV, F32, ctx, _name_the_case  # noqa: F401  (fixtures among them)

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- numbers that are not finite
@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,classes,dim,bad", [(70, 33, 30, [32]), (70, 64, 100, list(range(32, 64))), (70, 40, 200, list(range(32, 40))), (70, 64, 300, list(range(32, 64))),
                                               (70, 33, 30, [0]), (70, 20, 30, [19]), (70, 64, 100, list(range(32))), (70, 50, 30, [40]), (70, 2, 30, [0, 1]),
                                               (70, 65, 30, [64]), (70, 300, 200, [299]), (70, 300, 300, [0]), (20, 300, 100, [299]), (20, 300, 100, list(range(288, 300)))])
def test_classes_whose_weight_is_not_a_number(ctx, dtype, n, classes, dim, bad):  # noqa: F811
    """Each row's z has a NaN: neither its lse nor its loss is finite, wherever the class lies; rows that do not count stay 0."""
    rng = np.random.default_rng(n + classes + dim)
    x, w, labels = inputs(rng, n, classes, dim, dtype)
    for value in ([float("nan"), float("inf")] if dtype == F32 else [float("nan")]):           # (an infinity among 32-bit numbers gives NaN)
        w[bad, 3] = value
        counts = torch.from_numpy((labels >= 0) & (labels < classes)).to(DEV)
        loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        ctx.cross_entropy(x, n, dim, w, classes, on_gpu(labels), loss, lse)
        assert not bool(torch.isfinite(loss[counts]).any()) and not bool(torch.isfinite(lse[counts]).any())
        assert bool((loss[~counts] == 0).all()) and bool((lse[~counts] == 0).all())
