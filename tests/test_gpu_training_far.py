"""The training step's operators on an MI355X where numbers are near the ends of the 32-bit range."""
import numpy as np
import pytest
import torch

import training_reference as ref
from test_gpu_training_ops import DEV, F32, _name_the_case, check, check_norm_grad, ctx, f64     # noqa: F401  (fixtures among them)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("dtype", [F32, torch.bfloat16])
@pytest.mark.parametrize("dim", [1, 3, 8, 17, 64, 100, 255, 602, 1000, 1025, 2049])
def test_layer_norm_gradient_of_rows_far_from_zero(ctx, dtype, dim, given):
    """Rows without spread whose mean over their deviation (2^130) leaves the 32-bit range: x less the mean is 0, so that h is 0 and the gradient is
    rstd (g - mean(g)).  Every sum of the forward pass is exact, and so is the mean."""
    rng = np.random.default_rng(dim)
    n, far = 9, [0, 3, 4, 8]
    near = [i for i in range(n) if i not in far]
    x = torch.from_numpy(rng.normal(size=(n, dim)) * 1.5 + rng.normal(size=(n, 1))).to(dtype)
    for i in far:
        x[i] = 1.5 * 2.0 ** 110 * (-1) ** i
    dy = torch.from_numpy(rng.normal(size=(n, dim)) * 0.1).to(dtype)
    gamma = torch.from_numpy(rng.normal(size=dim)).float() if given else None
    g64 = f64(gamma) if given else np.ones(dim)
    there = gamma.to(DEV) if given else None
    y, mean, rstd = torch.empty(n, dim, dtype=dtype, device=DEV), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    ctx.layer_norm(x.to(DEV), n, dim, there, None, 1e-12, y, mean, rstd)
    assert np.array_equal(f64(mean)[far], f64(x)[far, 0]) and bool((y[far] == 0).all()) and bool((rstd[far] > 9e5).all())
    dx, dg, db = torch.empty(n, dim, dtype=dtype, device=DEV), torch.empty(dim, device=DEV), torch.empty(dim, device=DEV)
    ctx.layer_norm_grad(dy.to(DEV), x.to(DEV), n, dim, there, mean, rstd, dx, dg, db)
    m, s, x64, dy64 = f64(mean), f64(rstd), f64(x), f64(dy)
    want, _, _ = ref.layer_norm_grad(dy64[far], x64[far], g64, m[far], s[far])
    g = np.abs(dy64[far] * g64)
    u = 2.0 ** -24 * (8.0 + 4.0 * np.sqrt(dim))
    check(dx[far], want, 2 * s[far, None] * u * (g + g.mean(1, keepdims=True)) + ref.stored(want, dtype), "dx")
    check_norm_grad(dx[near], dg, None, dy64[near], x64[near], g64, m[near], s[near], dtype)      # (the far rows add 0 to dgamma)
    check_norm_grad(None, None, db, dy64, x64, g64, m, s, dtype)


@pytest.mark.parametrize("dtype", [F32, torch.bfloat16])
@pytest.mark.parametrize("largest,most", [(1e30, 1e-30), (3e38, 1e-37), (2.0 ** 100, 2.0 ** -91), (2.0 ** 127, 2.0 ** -126), (1e38, 3e-41), (1e25, 1e-20), (1e12, 1e-12)])
def test_clip_of_norms_far_beyond_the_largest_wanted(ctx, dtype, largest, most):
    """Factors down to 2^-270: each number within the formula's roundings, or half of the smallest 32-bit number twice where results are below 2^-126."""
    from paper_2505_10806_amd import binding as B
    rng = np.random.default_rng(int(np.log2(largest)))
    grads = [torch.from_numpy(rng.uniform(-1, 1, k) * largest * 2.0 ** -rng.integers(0, 60, k)).to(dtype) for k in (1, 7, 1000, 4099)]
    grads[0][0] = largest
    most = float(np.float32(most))
    norm64, want = ref.clip([f64(g) for g in grads], most)
    norm, out = torch.empty(1, device=DEV), [torch.empty(g.shape, dtype=dtype, device=DEV) for g in grads]
    ctx.clip_grad_norm(B.TensorList([g.to(DEV) for g in grads], out), most, norm)
    for o, w in zip(out, want):
        check(o, w, 2.0 ** -22 * np.abs(w) + 2.0 ** -149 + ref.stored(w, dtype), "clipped")
