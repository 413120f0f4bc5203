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


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("dim,out", [(64, 40), (64, 70), (256, 70)])
@pytest.mark.parametrize("scale,size", [(0, 0), (1, 60), (2, 125), (20, 100), (60, 60), (127, 0), (200, -60), (245, -115), (252, -120), (252, -24), (60, -60), (127, -126), (127, -130)])
def test_gradient_of_far_scales(ctx, dtype, dim, out, scale, size):
    """Scale bytes from the first to the largest that quantisation makes, times dy of 2^size.  A 32-bit number of dy counts as the next multiple of 2^-133
    towards 0; results below 2^-126 have roundings of 2^-149 each."""
    if dtype == torch.float16 and not -24 <= size <= 15:
        size = max(-24, min(15, size))
    if scale - 127 + size > 110:
        size = 0
    n = 200
    rng = np.random.default_rng(scale + 300 + size)
    groups = -(-dim // 32)
    packed = np.zeros((n, 4 * ref.words(dim)), dtype=np.uint8)
    packed[:, :16 * groups] = rng.integers(0, 256, size=(n, 16 * groups))
    packed[:, 16 * groups:17 * groups] = scale
    values = ref.dequantize(packed, dim)
    dy = torch.from_numpy(rng.uniform(-1.0, 1.0, (n, out)) * 2.0 ** size).to(dtype)
    grad = torch.empty(out, dim, device=DEV)
    ctx.mx4_matmul_grad(dy.to(DEV), torch.from_numpy(packed).view(F32).to(DEV), n, out, dim, grad)
    d = f64(dy)
    lost = 2.0 ** -133 * np.abs(values).sum(0)[None, :] if dtype == F32 else 0.0
    want = d.T @ values
    assert np.abs(want).max() < 2.0 ** 127
    check(grad, want, ref.sum_error(n, np.abs(d).T @ np.abs(values)) + lost + (4 * np.sqrt(n) + 8) * 2.0 ** -149, "grad")


def test_numbers_of_packed_rows_beyond_the_32_bit_range(ctx):
    """Scale bytes 253 and 254, which quantisation never makes: what leaves the 32-bit range reads as an infinity, and what that adds to a gradient is not finite;
    the product takes codes and scales as they are."""
    n, dim, out = 16, 32, 70
    packed = np.zeros((n, 20), dtype=np.uint8)
    packed[:, 0] = np.arange(n)                              # one number of each code to a row, the others 0
    packed[:, 16] = 252 + np.arange(n) % 3
    rows = torch.from_numpy(packed).view(F32).to(DEV)
    exact = ref.dequantize(packed, dim)
    with np.errstate(over="ignore"):
        read = exact.astype(np.float32)
    assert np.isposinf(read).any() and np.isneginf(read).any()
    back = torch.empty(n, dim, device=DEV)
    ctx.mx4_dequantize(rows, n, dim, back)
    assert np.array_equal(back.cpu().numpy(), read)
    weight = np.zeros((out, 20), dtype=np.uint8)
    weight[:, 0], weight[:, 16] = 2, 27                      # 2^-100
    y = torch.empty(n, out, device=DEV)
    ctx.mx4_matmul(rows, n, torch.from_numpy(weight).view(F32).to(DEV), out, dim, y)
    assert np.array_equal(f64(y), exact @ ref.dequantize(weight, dim).T)
    for outs in (out, 40):
        for i in range(n):
            grad = torch.empty(outs, dim, device=DEV)
            dy = torch.full((1, outs), 2.0 ** -100, device=DEV)
            ctx.mx4_matmul_grad(dy, rows[i:i + 1], 1, outs, dim, grad)
            finite = np.isfinite(read[i])
            assert np.array_equal(f64(grad)[:, finite], np.broadcast_to(exact[i, finite] * 2.0 ** -100, (outs, int(finite.sum()))))
            assert not np.isfinite(f64(grad)[:, ~finite]).any()
