"""Softmax cross entropy and its gradients on an MI355X where a row or a class stands far from the others."""
import numpy as np
import pytest
import torch

import training_reference as ref
import vector_reference as vec
from test_gpu_loss_ops import check_grads, inputs, on_gpu
from test_gpu_training_ops import DEV, F32, PAD, check, ctx, f64, _name_the_case  # noqa: F401  (fixtures among them)

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


# ---------------------------------------------------------------- shares of very different size
@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,classes,dim", [(100, 41, 30), (100, 64, 100), (100, 20, 200), (40, 33, 300), (3000, 41, 30), (100, 65, 30), (100, 300, 200)])
@pytest.mark.parametrize("far", [float("inf"), float("-inf"), 2.0 ** 126, 2.0 ** 40, 2.0 ** 20])
def test_a_row_goes_by_its_own_share(ctx, dtype, n, classes, dim, far):  # noqa: F811
    """One row's dloss is infinite or much larger: the others' dx are what they are without it, bit for bit, and within the bounds."""
    rng = np.random.default_rng(n + classes + dim)
    x, w, labels = inputs(rng, n, classes, dim, dtype)
    labels = np.clip(labels, 0, classes - 1)
    _, lse64 = vec.cross_entropy(vec.logits(f64(x), f64(w)), labels)
    lse = torch.from_numpy(lse64).float().to(DEV)
    dloss = torch.from_numpy(rng.normal(size=n) * np.exp2(rng.integers(-12, 8, n))).float().to(DEV)
    dloss[5] = 0.0
    dx, dw = torch.empty(n, dim, dtype=dtype, device=DEV), torch.empty(classes, dim, dtype=dtype, device=DEV)
    ctx.cross_entropy_grad(x, n, dim, w, classes, on_gpu(labels), lse, dx, dw, dloss=dloss, scale=0.5)
    check_grads(dx, dw, f64(x), f64(w), labels, f64(lse), f64(dloss) * 0.5, dtype)
    dloss[7] = far
    for with_weight in (True, False):
        again = torch.empty_like(dx)
        ctx.cross_entropy_grad(x, n, dim, w, classes, on_gpu(labels), lse, again, dw if with_weight else None, dloss=dloss, scale=0.5)
        rest = np.delete(np.arange(n), 7)
        at = torch.from_numpy(rest).to(DEV)
        check_grads(again[at], None, f64(x)[rest], f64(w), labels[rest], f64(lse)[rest], f64(dloss)[rest] * 0.5, dtype)
        assert torch.equal(again[at], dx[at])
    if not np.isfinite(far):
        assert not bool(torch.isfinite(again[7]).any()) and not bool(torch.isfinite(dw).any())


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,classes,dim", [(200, 41, 30), (200, 64, 100), (200, 20, 200), (64, 33, 300), (200, 65, 30)])
def test_small_shares_keep_their_bits(ctx, dtype, n, classes, dim):  # noqa: F811
    """Shares down to 2^-100 of the largest (of f16: 2^-38, with a scale that brings the smallest dx into its range), each dx within its own row's bounds;
    a class far below the others keeps a small g in every row."""
    rng = np.random.default_rng(n + classes + dim)
    x, w, labels = inputs(rng, n, classes, dim, dtype, spread=0.5)
    labels = np.clip(labels, 0, classes - 1)
    down, scale = (38, 2.0 ** 24) if dtype == torch.float16 else (100, 1.0)
    _, lse64 = vec.cross_entropy(vec.logits(f64(x), f64(w)), labels)
    lse = torch.from_numpy(lse64).float().to(DEV)
    dloss = torch.from_numpy(rng.uniform(0.5, 1.0, n) * np.exp2(-rng.integers(down - 20, down + 1, n))).float().to(DEV)
    dloss[0] = 1.0
    dx, dw = torch.empty(n, dim, dtype=dtype, device=DEV), torch.empty(classes, dim, dtype=dtype, device=DEV)
    ctx.cross_entropy_grad(x, n, dim, w, classes, on_gpu(labels), lse, dx, dw, dloss=dloss, scale=scale)
    rest = np.arange(1, n)
    check_grads(dx[1:], None, f64(x)[rest], f64(w), labels[rest], f64(lse)[rest], f64(dloss)[rest] * scale, dtype)


# ---------------------------------------------------------------- logits of any size
@pytest.mark.parametrize("dtype,far", [(F32, 10), (F32, 33), (F32, 60), (F32, 127), (torch.bfloat16, 10), (torch.bfloat16, 33), (torch.bfloat16, 60), (torch.bfloat16, 127),
                                       (torch.float16, 10), (torch.float16, 30)])
@pytest.mark.parametrize("n,classes,dim", [(100, 40, 64), (100, 33, 300), (20, 300, 64), (100, 300, 64), (100, 300, 16), (100, 200, 200), (100, 300, 300), (700, 5000, 64), (700, 5000, 300)])
def test_logits_of_any_size(ctx, dtype, far, n, classes, dim):  # noqa: F811
    """z of one product each, exact: m 2^(far - 1) with whole m in [-3, 3].  exp(z - lse) is 0 below a row's largest (its exponent is -512 or less).  lse = m + log(count):
    one rounding to 32 bits, one of m / ln 2, two steps of log(count) < 9.  Given the largest z as lse, p is 1 or 0, so that sums of whole numbers below 2^13 times
    powers of two make both gradients exact up to their storing; where lse is small (far 10) p may err as lse / ln 2 does."""
    rng = np.random.default_rng(far + classes)
    left = far // 2
    x = torch.zeros(n, dim, dtype=dtype, device=DEV)
    at = rng.integers(0, dim, n)
    x[torch.arange(n), torch.from_numpy(at)] = 2.0 ** left
    whole = rng.integers(-3, 4, size=(classes, dim))
    whole[:, ::2] = -np.abs(whole[:, ::2]) - (whole[:, ::2] == 0)                   # (columns whose largest is below zero too)
    whole[:, 3] = np.where(np.arange(classes) == classes // 2, 3, -3)               # (and one whose largest stands alone)
    w = (torch.from_numpy(whole).double() * 2.0 ** (far - 1 - left)).to(dtype).to(DEV)
    labels = rng.integers(0, classes, n)
    labels[:n // 2] = whole[:, at[:n // 2]].argmax(0)
    labels[3] = -1
    counts = labels >= 0
    z = f64(x) @ f64(w).T
    want, want_lse = vec.cross_entropy(z, labels)
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    ctx.cross_entropy(x, n, dim, w, classes, on_gpu(labels), loss, lse)
    allowed = 2.0 ** -23 * np.abs(want_lse) + 2.0 ** -19
    with np.errstate(over="ignore"):
        stored = want.astype(np.float32).astype(np.float64)                           # (the distance of two z may be beyond 32 bits)
    check(lse, want_lse, allowed, "lse")
    check(loss, np.where(np.isinf(stored), stored, want), 2 * allowed + 2.0 ** -23 * np.abs(want), "loss")
    dx, dw = torch.empty(n, dim, dtype=dtype, device=DEV), torch.empty(classes, dim, dtype=dtype, device=DEV)
    saved = torch.from_numpy(np.where(counts, z.max(1), 0.0)).float().to(DEV)
    ctx.cross_entropy_grad(x, n, dim, w, classes, on_gpu(labels), saved, dx, dw, scale=2.0 ** -12)
    want_dx, want_dw, p, g = vec.cross_entropy_grad(z, labels, f64(saved), np.full(n, 2.0 ** -12), f64(x), f64(w))
    if far == 10:
        eg = 2.0 ** -12 * p * 2.0 ** -22 * (np.abs(z) + np.abs(f64(saved))[:, None] + 2.0)
        eg += np.abs(g) * (ref.HALF_ULP[dtype] if dtype != F32 else 2.0 ** -20)
        eg += 2.0 ** -50 if dtype == torch.float16 else 0.0                           # (f16's smallest step, 2^-38 of the share)
    else:
        eg = np.zeros_like(p)
    check(dx, want_dx, eg @ np.abs(f64(w)) + (ref.stored(want_dx, dtype) if dtype != F32 or far == 10 else 2.0 ** -149), "dx")
    check(dw, want_dw, eg.T @ np.abs(f64(x)) + (ref.stored(want_dw, dtype) if dtype != F32 or far == 10 else 2.0 ** -149), "dweight")


# ---------------------------------------------------------------- many classes beside one
@pytest.mark.parametrize("dtype,n,dim", [(torch.bfloat16, 33_000, 100), (torch.bfloat16, 33_000, 200), (torch.bfloat16, 33_000, 300), (torch.float16, 4096, 64), (F32, 33_000, 100),
                                         (F32, 33_000, 200), (F32, 4096, 300), (torch.bfloat16, 4096, 300), (F32, 32, 100), (torch.bfloat16, 8, 100)])
def test_what_one_class_leaves_is_shared_by_many(ctx, dtype, n, dim):  # noqa: F811
    """A class of z = a against 232964 of z = 0: lse = a + log(1 + c), c = 232964 e^-a.  Roundings of lse's size: a / ln 2, the log's two steps, lse itself; of 1: up to
    sixteen additions beside the one class, four of parts, exp2's step: together below 8 steps of 2^-24 (a + 1) (16 <= a + 1).  What the many add: 2^-18 of c."""
    classes = 232_965
    x, w = torch.zeros(n, dim, dtype=dtype, device=DEV), torch.zeros(classes, dim, dtype=dtype, device=DEV)
    w[:, 1] = 3.0                                          # (against zeros of x)
    first = torch.tensor([3.0, 3.25, 3.5, 4.0], device=DEV)[torch.arange(n, device=DEV) % 4]
    x[:, 0] = first.to(dtype)
    for label in (0, 64, 133, 116_000):
        w[:, 0] = 0.0
        w[label, 0] = 5.0
        at = torch.full((n,), label, dtype=torch.int32, device=DEV)
        loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        ctx.cross_entropy(x, n, dim, w, classes, at, loss, lse)
        a = first.double() * 5.0
        c = (classes - 1) * torch.exp(-a)
        want = torch.log1p(c)
        allowed = 8 * 2.0 ** -24 * (a + 1.0) + 2.0 ** -18 * c
        assert bool(((lse.double() - a - want).abs() <= allowed).all()) and bool(((loss.double() - want).abs() <= allowed).all())


# ---------------------------------------------------------------- long sums in 32 bits
def one_sign(gen, rows, dim):
    return torch.randn(rows, dim, generator=gen, device=DEV) * 0.2 + 1.0


def long_sum(count, size):
    """A sum of `count` terms in stretches of 4096: of each, and of their sums."""
    return ref.sum_error(min(count, 4096), size) + ref.sum_error(-(-count // 4096), size)


def g_error(p, z, x, w, lse, share):
    return share * p * (ref.sum_error(x.shape[1], np.abs(x) @ np.abs(w).T) + 2.0 ** -20 * (np.abs(x) @ np.abs(w).T) + 2.0 ** -22 * (np.abs(z) + np.abs(lse)[:, None] + 2.0))


@pytest.mark.parametrize("n,classes,dim", [(200_000, 66_000, 16), (70_000, 66_000, 40), (1_000_000, 1000, 16), (1_000_003, 47, 16), (60_000, 70_000, 300)])
def test_weight_gradients_of_many_rows_of_one_sign(ctx, n, classes, dim):  # noqa: F811
    """f32: a sum of many numbers of one sign, half of it taken away again by the label's rows, errs as sums of 4096 do."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(n)
    x, w = one_sign(gen, n, dim), torch.randn(classes, dim, generator=gen, device=DEV) * 0.1
    labels = torch.randint(0, classes, (n,), generator=gen, device=DEV).int()
    lse = torch.empty(n, device=DEV)
    ctx.cross_entropy(x, n, dim, w, classes, labels, None, lse)
    dw = torch.full((classes + 1, dim), PAD, device=DEV)
    ctx.cross_entropy_grad(x, n, dim, w, classes, labels, lse, None, dw[:classes])
    assert bool((dw[classes] == PAD).all())
    some = np.unique(np.r_[0:12, classes - 12:classes])
    at = torch.from_numpy(some).to(DEV)
    x64, w64, l64, told = f64(x), f64(w[at]), f64(lse), labels.long().cpu().numpy()
    z = x64 @ w64.T
    p = np.exp(z - l64[:, None])
    g = p - (told[:, None] == some[None, :])
    eg = g_error(p, z, x64, w64, l64, 1.0) + np.abs(g) * (2.0 ** -23 + 2.0 ** -20)
    check(dw[at], g.T @ x64, eg.T @ np.abs(x64) + long_sum(n, np.abs(g).T @ np.abs(x64)), "dweight")


@pytest.mark.parametrize("n,classes,dim", [(33_000, 400_000, 16), (33_000, 100_000, 100), (4096, 300_000, 300), (2000, 1_000_000, 16)])
def test_row_gradients_against_many_classes_of_one_sign(ctx, n, classes, dim):  # noqa: F811
    gen = torch.Generator(device=DEV)
    gen.manual_seed(n)
    x, w = torch.randn(n, dim, generator=gen, device=DEV) * 0.1, one_sign(gen, classes, dim)
    labels = torch.randint(0, classes, (n,), generator=gen, device=DEV).int()
    lse = torch.empty(n, device=DEV)
    ctx.cross_entropy(x, n, dim, w, classes, labels, None, lse)
    dx = torch.full((n + 1, dim), PAD, device=DEV)
    ctx.cross_entropy_grad(x, n, dim, w, classes, labels, lse, dx[:n], None)
    assert bool((dx[n] == PAD).all())
    some = np.unique(np.r_[0:12, n - 12:n])
    at = torch.from_numpy(some).to(DEV)
    x64, w64, l64, told = f64(x[at]), f64(w), f64(lse[at]), labels[at].long().cpu().numpy()
    z = x64 @ w64.T
    p = np.exp(z - l64[:, None])
    g = p.copy()
    g[np.arange(len(some)), told] -= 1.0
    eg = g_error(p, z, x64, w64, l64, 1.0) + np.abs(g) * (2.0 ** -23 + 2.0 ** -20)
    check(dx[at], g @ w64, eg @ np.abs(w64) + long_sum(classes, np.abs(g) @ np.abs(w64)), "dx")


@pytest.mark.parametrize("n,classes,dim", [(64, 200, 8192), (64, 100, 20_000), (33, 65, 65_536), (5, 40, 8191)])
def test_long_rows_of_one_sign(ctx, n, classes, dim):  # noqa: F811
    """f32: z of many numbers of one sign errs as sums of 128 do, and each row's loss and gradients with it."""
    rng = np.random.default_rng(dim)
    x = torch.from_numpy(rng.random((n, dim))).float().to(DEV)
    w = torch.from_numpy(rng.random((classes, dim)) * (400.0 / dim)).float().to(DEV)
    labels = rng.integers(0, classes, n)
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    ctx.cross_entropy(x, n, dim, w, classes, on_gpu(labels), loss, lse)
    x64, w64 = f64(x), f64(w)
    z = vec.logits(x64, w64)
    size = np.abs(x64) @ np.abs(w64).T
    # (chunks' sums are added with roundings to the nearest, 2^-24 each, independent: four deviations)
    ez = 2.0 ** -20 * size + ref.sum_error(128, size) + 4.0 * np.sqrt(dim / 128) * 2.0 ** -24 * size
    want, want_lse = vec.cross_entropy(z, labels)
    allowed = ez.max(1) + 2.0 ** -22 * (np.abs(z).max(1) + np.abs(want_lse) + 2.0) + ref.sum_error(classes, 1.0)
    check(lse, want_lse, allowed, "lse")
    check(loss, want, allowed + ez.max(1) + 2.0 ** -23 * np.abs(want), "loss")
    lse = torch.from_numpy(want_lse).float().to(DEV)
    dx, dw = torch.empty(n, dim, device=DEV), torch.empty(classes, dim, device=DEV)
    ctx.cross_entropy_grad(x, n, dim, w, classes, on_gpu(labels), lse, dx, dw)
    want_dx, want_dw, p, g = vec.cross_entropy_grad(z, labels, f64(lse), np.ones(n), x64, w64)
    eg = p * (ez + 2.0 ** -22 * (np.abs(z) + np.abs(f64(lse))[:, None] + 2.0)) + np.abs(g) * (2.0 ** -23 + 2.0 ** -20)
    check(dx, want_dx, eg @ np.abs(w64) + ref.sum_error(classes, np.abs(g) @ np.abs(w64)) + ref.stored(want_dx, F32), "dx")
    check(dw, want_dw, eg.T @ np.abs(x64) + ref.sum_error(n, np.abs(g).T @ np.abs(x64)) + ref.stored(want_dw, F32), "dweight")
