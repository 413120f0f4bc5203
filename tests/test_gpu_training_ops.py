"""The training step's operators on an MI355X against their 64-bit forms (tests/training_reference.py), at the sizes, strides, counts and
values where they can go wrong."""
import numpy as np
import pytest
import torch

import training_reference as ref
from gpu_common import log

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32 = torch.float32
PAD = -77.0                     # what lies behind and between rows


@pytest.fixture(scope="module")
def ctx():
    from paper_2505_10806_amd import binding as B
    c = B.Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


@pytest.fixture(autouse=True)
def _name_the_case(request):
    log(f"[training] {request.node.name}")
    yield
    torch.cuda.synchronize()


def f64(t):
    return t.detach().double().cpu().numpy()


def padded(values, dtype, extra=0, offset=0):
    """A cuda view [n, dim] of the values whose rows lie `extra` numbers apart, `offset` numbers into an allocation full of PAD."""
    values = torch.as_tensor(values)
    n, dim = values.shape
    stride = dim + extra
    flat = torch.full((offset + n * stride + 8,), PAD, dtype=dtype, device=DEV)
    view = torch.as_strided(flat, (n, dim), (stride, 1), offset)
    view.copy_(values.to(dtype))
    return flat, view


def untouched(flat, view):
    """Everything outside the view still holds PAD."""
    mark = torch.ones_like(flat, dtype=torch.bool)
    torch.as_strided(mark, view.shape, view.stride(), view.storage_offset()).fill_(False)
    return bool((flat[mark] == PAD).all())


def to_packed(bytes_, extra=0):
    """float32 [n, words (+ extra)] on the GPU of packed bytes."""
    n, size = bytes_.shape
    out = torch.full((n, size // 4 + extra), PAD, dtype=F32, device=DEV)
    out[:, :size // 4] = torch.from_numpy(bytes_.copy()).view(torch.uint8).view(F32).to(DEV).view(n, size // 4)
    return out


def of_packed(t, dim):
    return np.ascontiguousarray(t.cpu().contiguous().view(torch.uint8).numpy()[:, :4 * ref.words(dim)])


def check(got, want, allowed, what):
    got = f64(got) if isinstance(got, torch.Tensor) else got
    bad = ~(np.abs(got - want) <= allowed)
    bad &= ~((got == want) | (np.isnan(got) & np.isnan(want)))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off; first {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}, " \
                          f"{np.broadcast_to(allowed, want.shape)[bad][0]} allowed"


def packed_rows(rng, n, dim, spread=4):
    """Packed bytes of normal rows whose groups differ in size."""
    x = rng.normal(size=(n, dim)) * np.exp2(rng.integers(-spread, spread + 1, size=(n, 1)))
    return ref.quantize(x.astype(np.float32).astype(np.float64))


# ---------------------------------------------------------------- 4-bit rows
@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,dim,extra,offset", [(1, 1, 0, 0), (3, 31, 0, 1), (2, 32, 5, 0), (5, 33, 0, 3), (7, 64, 0, 0), (130, 100, 0, 0), (37, 127, 1, 1),
                                                (64, 128, 0, 0), (33, 129, 3, 2), (1025, 256, 0, 0), (17, 602, 0, 0), (9, 1024, 6, 5), (3, 65536, 0, 0)])
def test_quantize_and_back_are_exact(ctx, dtype, n, dim, extra, offset):
    rng = np.random.default_rng(n * 1000 + dim)
    x = torch.from_numpy(rng.normal(size=(n, dim)) * np.exp2(rng.integers(-20, 8, size=(n, 1)))).to(dtype)
    flat, view = padded(x, dtype, extra, offset)
    want, values = ref.quantize(f64(x))
    words = ref.words(dim)
    packed = torch.full((n, words + extra), PAD, dtype=F32, device=DEV)
    ctx.mx4_quantize(view, n, dim, packed)
    torch.cuda.synchronize()
    assert np.array_equal(of_packed(packed, dim), want)
    assert bool((packed[:, words:] == PAD).all()) and untouched(flat, view)
    flat, back = padded(torch.zeros(n, dim), dtype, extra, offset)
    ctx.mx4_dequantize(packed, n, dim, back)
    torch.cuda.synchronize()
    rounded = torch.from_numpy(values).float().to(dtype)
    assert torch.equal(back.cpu(), rounded) and untouched(flat, back)


@pytest.mark.parametrize("dtype", ref.TYPES)
def test_quantize_extremes(ctx, dtype):
    x = torch.zeros(12, 96, dtype=dtype)
    big = torch.finfo(dtype).max
    x[0, 5], x[0, 70] = big, -big
    x[1, 0], x[1, 33] = float("inf"), 1.0
    x[2, 31], x[2, 64] = float("nan"), -2.0
    x[3, 95], x[3, 0] = -float("inf"), float("nan")
    x[4, :32] = torch.finfo(dtype).tiny
    x[5, 40] = 2.0 ** -24 if dtype == torch.float16 else 2.0 ** -133
    x[6] = -0.0
    x[7, :8] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], dtype=dtype)
    x[8, :8] = -x[7, :8]
    x[9, :3] = torch.tensor([4.0, 7.875, -7.5], dtype=dtype)
    x[10] = torch.arange(96, dtype=torch.float32).to(dtype) - 48
    want, values = ref.quantize(f64(x))
    packed = torch.zeros(12, ref.words(96), device=DEV)
    ctx.mx4_quantize(x.to(DEV), 12, 96, packed)
    assert np.array_equal(of_packed(packed, 96), want)
    back = torch.empty(12, 96, device=DEV)
    ctx.mx4_dequantize(packed, 12, 96, back)
    assert np.array_equal(f64(back), values, equal_nan=True)


def test_every_scale_and_code_of_a_packed_row_is_read(ctx):
    packed = np.zeros((256, 20), dtype=np.uint8)
    packed[:, :16] = np.arange(256, dtype=np.uint8).reshape(16, 16)[np.arange(256) % 16]
    packed[:, 16] = np.arange(256)
    rows = to_packed(packed)
    want = ref.dequantize(packed, 32)
    for dtype in ref.TYPES:
        back = torch.empty(256, 32, dtype=dtype, device=DEV)
        ctx.mx4_dequantize(rows, 256, 32, back)
        assert np.array_equal(f64(back), f64(torch.from_numpy(want).float().to(dtype)), equal_nan=True)


def test_room_for_far_more_rows_than_there_are(ctx):
    """A count of rows up to the largest that is allowed beside a small one on the device: what a workgroup works on does not grow with it."""
    from paper_2505_10806_amd import binding as B
    rng = np.random.default_rng(5)
    live, dim = 40, 65_532
    x = torch.from_numpy(rng.normal(size=(live, dim))).float()
    want, values = ref.quantize(f64(x))
    n_dev = torch.tensor([live], dtype=torch.int32, device=DEV)
    most = (1 << 31) - 1
    packed, back = torch.full((live, ref.words(dim)), PAD, device=DEV), torch.full((live, dim), PAD, device=DEV)
    there = x.to(DEV)
    stream = torch.cuda.current_stream().cuda_stream
    assert B._lib.rg_mx4_quantize(ctx._h, there.data_ptr(), 0, dim, most, n_dev.data_ptr(), dim, packed.data_ptr(), ref.words(dim), stream) == 0
    assert np.array_equal(of_packed(packed, dim), want)
    assert B._lib.rg_mx4_dequantize(ctx._h, packed.data_ptr(), ref.words(dim), most, n_dev.data_ptr(), dim, back.data_ptr(), 0, dim, stream) == 0
    assert np.array_equal(f64(back), values)


@pytest.mark.parametrize("live", [0, 1, 20, 50, 51])
def test_counts_on_the_device(ctx, live):
    """Every operator works on min(n, *n_dev) rows and leaves the others alone."""
    rng = np.random.default_rng(live)
    n, dim, out = 50, 70, 24
    real = min(n, live)
    n_dev = torch.tensor([live], dtype=torch.int32, device=DEV)
    x = torch.from_numpy(rng.normal(size=(n, dim))).float()
    want, values = ref.quantize(f64(x))
    packed = torch.full((n, ref.words(dim)), PAD, device=DEV)
    ctx.mx4_quantize(x.to(DEV), n, dim, packed, n_dev=n_dev)
    assert np.array_equal(of_packed(packed, dim)[:real], want[:real]) and bool((packed[real:] == PAD).all())
    back = torch.full((n, dim), PAD, device=DEV)
    rows = to_packed(want)
    ctx.mx4_dequantize(rows, n, dim, back, n_dev=n_dev)
    assert np.array_equal(f64(back)[:real], values[:real]) and bool((back[real:] == PAD).all())
    wb, wv = packed_rows(rng, out, dim)
    y = torch.full((n, out), PAD, device=DEV)
    ctx.mx4_matmul(rows, n, to_packed(wb), out, dim, y, n_dev=n_dev)
    check(y[:real], values[:real] @ wv.T, sum_allowed(dim, values[:real], wv), "y")
    assert bool((y[real:] == PAD).all())
    dy = torch.from_numpy(rng.normal(size=(n, out))).float()
    dy[real:] = float("nan")
    poisoned = want.copy()
    poisoned[real:, 16 * 3:16 * 3 + 3] = 255
    grad = torch.full((out, dim), PAD, device=DEV)
    ctx.mx4_matmul_grad(dy.to(DEV), to_packed(poisoned), n, out, dim, grad, n_dev=n_dev)
    d = f64(dy)[:real]
    check(grad, d.T @ values[:real], ref.sum_error(real, np.abs(d).T @ np.abs(values[:real])), "grad")
    xn = x.clone()
    xn[real:] = float("nan")
    yn, mean, rstd = (torch.full(s, PAD, device=DEV) for s in ((n, dim), (n,), (n,)))
    ctx.layer_norm(xn.to(DEV), n, dim, None, None, 1e-5, yn, mean, rstd, n_dev=n_dev)
    assert bool((yn[real:] == PAD).all() and (mean[real:] == PAD).all() and (rstd[real:] == PAD).all())
    check_norm(yn[:real], mean[:real], rstd[:real], f64(x)[:real], np.ones(dim), np.zeros(dim), 1e-5, F32)
    dx, dg, db = torch.full((n, dim), PAD, device=DEV), torch.full((dim,), PAD, device=DEV), torch.full((dim,), PAD, device=DEV)
    dyn = torch.from_numpy(rng.normal(size=(n, dim))).float()
    dyn[real:] = float("nan")
    ctx.layer_norm_grad(dyn.to(DEV), xn.to(DEV), n, dim, None, mean, rstd, dx, dg, db, n_dev=n_dev)
    assert bool((dx[real:] == PAD).all())
    check_norm_grad(dx[:real], dg, db, f64(dyn)[:real], f64(x)[:real], np.ones(dim), f64(mean)[:real], f64(rstd)[:real], F32)


# ---------------------------------------------------------------- product
def sum_allowed(dim, a, b, dtype=F32):
    size = np.abs(a) @ np.abs(b).T
    return ref.sum_error(dim, size) + ref.stored(a @ b.T, dtype)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,dim,out", [(1, 1, 1), (1, 602, 41), (2, 32, 16), (15, 33, 17), (16, 128, 16), (17, 129, 15), (31, 100, 47), (64, 64, 64), (65, 160, 130),
                                       (256, 256, 256), (257, 256, 256), (300, 602, 41), (1000, 100, 128), (513, 1024, 72), (129, 2100, 33), (3961, 64, 512),
                                       (5, 65536, 3), (700, 17, 1000), (40_001, 100, 3), (70_001, 128, 200)])
def test_product(ctx, dtype, n, dim, out):
    rng = np.random.default_rng(n + dim * 7 + out)
    rb, rv = packed_rows(rng, n, dim)
    wb, wv = packed_rows(rng, out, dim)
    extra = n % 3                                        # packed rows of one word's alignment, and of 16 bytes'
    flat, y = padded(torch.zeros(n, out), dtype, out % 5, n % 2)
    ctx.mx4_matmul(to_packed(rb, extra), n, to_packed(wb, out % 4), out, dim, y)
    torch.cuda.synchronize()
    check(y, rv @ wv.T, sum_allowed(dim, rv, wv, dtype), "y")
    assert untouched(flat, y)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,dim,out", [(4096, 256, 250), (4097, 256, 250), (1600, 602, 250), (1650, 602, 250), (500, 1024, 500), (20, 1100, 1030),
                                       (300, 2050, 600), (5000, 1100, 70), (20_000, 1056, 19), (30_001, 33, 65), (12_000, 602, 41), (9001, 300, 130),
                                       (6000, 513, 72), (4100, 1024, 72), (10_001, 800, 300), (140_000, 100, 1), (70_000, 31, 23)])
def test_product_of_many_sizes(ctx, dtype, n, dim, out):
    """Few rows and many, rows that registers hold and longer ones, results with gaps between their rows and without."""
    rng = np.random.default_rng(n + dim + out)
    xb, xv = packed_rows(rng, n, dim)
    wb, wv = packed_rows(rng, out, dim)
    flat, y = padded(torch.zeros(n, out), dtype, n % 2 * 3, n % 2)
    ctx.mx4_matmul(to_packed(xb), n, to_packed(wb), out, dim, y)
    torch.cuda.synchronize()
    check(y, xv @ wv.T, sum_allowed(dim, xv, wv, dtype), "y")
    assert untouched(flat, y)


def test_product_of_groups_that_are_not_numbers(ctx):
    """A NaN group of a row makes that row's results NaN and no other's; one of the weight, that output's."""
    rng = np.random.default_rng(5)
    for n, dim, out in ((40, 200, 40), (400, 200, 40)):
        rb, rv = packed_rows(rng, n, dim)
        wb, wv = packed_rows(rng, out, dim)
        groups = -(-dim // 32)
        rb[3, 16 * groups + 6] = 255                     # the ragged last group
        rb[17, 16 * groups] = 255
        wb[9, 16 * groups + 2] = 255
        rows, weight = to_packed(rb), to_packed(wb)
        want = ref.dequantize(rb, dim) @ ref.dequantize(wb, dim).T
        y = torch.empty(n, out, device=DEV)
        ctx.mx4_matmul(rows, n, weight, out, dim, y)
        assert np.array_equal(np.isnan(f64(y)), np.isnan(want))
        assert int(np.isnan(want).sum()) == 2 * out + n - 2
        ok = ~np.isnan(want)
        check(f64(y)[ok], want[ok], sum_allowed(dim, rv, wv)[ok], "y")


def test_product_of_far_scales(ctx):
    """Scales from 2^-127 to 2^125 whose products are ordinary numbers."""
    rng = np.random.default_rng(6)
    for shift in (-120, -60, 60, 115):
        rv0 = rng.normal(size=(33, 96)) * 2.0 ** shift
        wv0 = rng.normal(size=(20, 96)) * 2.0 ** -shift
        rb, rv = ref.quantize(rv0)
        wb, wv = ref.quantize(wv0)
        y = torch.empty(33, 20, device=DEV)
        ctx.mx4_matmul(to_packed(rb), 33, to_packed(wb), 20, 96, y)
        check(y, rv @ wv.T, sum_allowed(96, rv, wv), f"shift {shift}")


# ---------------------------------------------------------------- the weight's gradient
@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,dim,out", [(0, 40, 5), (1, 1, 1), (1, 602, 41), (31, 33, 17), (32, 128, 64), (33, 129, 65), (255, 100, 47), (257, 256, 256), (1000, 602, 41),
                                       (2049, 64, 3), (3961, 257, 130), (20_003, 100, 128), (50_001, 128, 258), (700, 17, 1000), (500, 2100, 9)])
def test_gradient(ctx, dtype, n, dim, out):
    rng = np.random.default_rng(n + dim * 7 + out)
    rb, rv = packed_rows(rng, max(n, 1), dim)
    rv = rv[:n]
    dy = torch.from_numpy(rng.normal(size=(max(n, 1), out)) * 0.01).to(dtype)
    flat_dy, vdy = padded(dy, dtype, n % 4, out % 2)
    flat, grad = padded(torch.zeros(out, dim), F32, dim % 3, 1)
    ctx.mx4_matmul_grad(vdy, to_packed(rb, n % 3), n, out, dim, grad)
    torch.cuda.synchronize()
    d = f64(dy)[:n]
    check(grad, d.T @ rv, ref.sum_error(n, np.abs(d).T @ np.abs(rv)), "grad")
    assert untouched(flat, grad)


@pytest.mark.parametrize("dtype", ref.TYPES)
def test_gradient_of_what_is_not_finite(ctx, dtype):
    """Infinities and NaN of dy reach their outputs only, as in the formula."""
    n, dim, out = 300, 140, 70
    rng = np.random.default_rng(8)
    rv0 = np.abs(rng.normal(size=(n, dim))) + 1.0
    rb, rv = ref.quantize(rv0)
    dy = torch.from_numpy(rng.normal(size=(n, out))).to(dtype)
    dy[7, 3], dy[100, 20], dy[299, 69] = float("inf"), -float("inf"), float("nan")
    rb[50, 16 * 5 + 4] = 255
    with np.errstate(invalid="ignore"):
        want = f64(dy).T @ ref.dequantize(rb, dim)
    grad = torch.empty(out, dim, device=DEV)
    ctx.mx4_matmul_grad(dy.to(DEV), to_packed(rb), n, out, dim, grad)
    got = f64(grad)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isposinf(got), np.isposinf(want))
    assert np.array_equal(np.isneginf(got), np.isneginf(want)) and np.isposinf(want).any() and np.isneginf(want).any()
    ok = np.isfinite(want)
    size = np.nan_to_num(np.abs(f64(dy)), posinf=0, nan=0).T @ np.nan_to_num(np.abs(rv))
    check(got[ok], want[ok], ref.sum_error(n, size)[ok], "grad")


def test_gradient_keeps_all_bits_of_dy(ctx):
    """Numbers with bits in every place, whose products with 1 are themselves: exact."""
    n, dim, out = 1, 32, 64
    bits = torch.arange(out, dtype=torch.int32) * 0x0135791 + 0x3F000001
    dy = bits.view(F32).clone()
    dy[1::2] *= -1
    dy[5], dy[6] = 2.0 ** -126, 3.4e38
    rb, _ = ref.quantize(np.ones((n, dim)))
    grad = torch.empty(out, dim, device=DEV)
    ctx.mx4_matmul_grad(dy.view(1, out).to(DEV), to_packed(rb), n, out, dim, grad)
    assert torch.equal(grad.cpu(), dy[:, None].expand(out, dim))
    half = torch.arange(0x0001, 0x7C00, 0x1F7, dtype=torch.int16).view(torch.float16)         # every exponent, subnormals among them
    grad = torch.empty(half.numel(), dim, device=DEV)
    ctx.mx4_matmul_grad(half.view(1, -1).to(DEV), to_packed(rb), 1, half.numel(), dim, grad)
    assert torch.equal(grad.cpu(), half.float()[:, None].expand(half.numel(), dim))


def test_gradient_is_the_difference_quotient_of_the_product(ctx):
    """The product is linear in the weight's numbers: moving one code changes sum(dy y) by the step times the gradient."""
    rng = np.random.default_rng(9)
    n, dim, out = 65, 70, 19
    rb, rv = packed_rows(rng, n, dim, 1)
    wb, wv = ref.quantize(rng.normal(size=(out, dim)))
    dy = torch.from_numpy(rng.normal(size=(n, out))).float()
    rows, y0, y1 = to_packed(rb), torch.empty(n, out, device=DEV), torch.empty(n, out, device=DEV)
    grad = torch.empty(out, dim, device=DEV)
    ctx.mx4_matmul(rows, n, to_packed(wb), out, dim, y0)
    ctx.mx4_matmul_grad(dy.to(DEV), rows, n, out, dim, grad)
    noise = sum_allowed(dim, rv, wv)
    for j, k in ((0, 0), (3, 31), (7, 32), (18, 69), (11, 64)):
        changed = wb.copy()
        place = k // 2
        changed[j, place] ^= 0x10 << 3 if k % 2 else 0x08                                    # the sign of the number
        step = ref.dequantize(changed, dim)[j, k] - wv[j, k]
        ctx.mx4_matmul(rows, n, to_packed(changed), out, dim, y1)
        moved = float(((f64(y1) - f64(y0)) * f64(dy)).sum())
        allowed = 2 * float((noise[:, j] * np.abs(f64(dy)[:, j])).sum()) + abs(step) * ref.sum_error(n, float(np.abs(f64(dy)[:, j]) @ np.abs(rv[:, k])))
        assert step != 0 or wv[j, k] == 0
        assert abs(moved - step * float(grad[j, k])) <= allowed


# ---------------------------------------------------------------- layer norm
def check_norm(y, mean, rstd, x, gamma, beta, eps, dtype):
    n, dim = x.shape
    if n == 0:
        return
    want, m, s = ref.layer_norm(x, gamma, beta, eps)
    top = np.abs(x).max(1, keepdims=True)
    u = 2.0 ** -24 * (8.0 + 4.0 * np.sqrt(dim))          # four deviations of a sum of dim numbers and eight roundings more
    # an error of the mean of u * top moves a number's distance from it by as much, and the variance's root by u top (relative to rstd)
    slack = u * top * s[:, None]
    h = (x - m[:, None]) * s[:, None]
    check(mean, m, u * top[:, 0], "mean")
    check(rstd, s, s * (u + 2 * slack[:, 0] ** 2 + 2 * slack[:, 0]), "rstd")
    allowed = np.abs(gamma) * (slack + np.abs(h) * (u + 2 * slack + 2 * slack ** 2)) + u * (np.abs(h * gamma) + np.abs(beta))
    check(y, want, allowed + ref.stored(want, dtype), "y")


def check_norm_grad(dx, dgamma, dbeta, dy, x, gamma, mean, rstd, dtype):
    n, dim = x.shape
    want, wg, wb = ref.layer_norm_grad(dy, x, gamma, mean, rstd)
    u = 2.0 ** -24 * (8.0 + 4.0 * np.sqrt(dim))
    h = (x - mean[:, None]) * rstd[:, None]
    eh = 2.0 ** -23 * 2 * (np.abs(h) + (np.abs(x) + np.abs(mean)[:, None]) * rstd[:, None])      # error of h: its three operations
    g = np.abs(dy * gamma)
    if dx is not None and n:
        along = (g * np.abs(h)).mean(1, keepdims=True)
        allowed = rstd[:, None] * (u * (g + g.mean(1, keepdims=True) + np.abs(h) * along) + eh * along + np.abs(h) * (g * eh).mean(1, keepdims=True))
        check(dx, want, 2 * allowed + ref.stored(want, dtype), "dx")
    if dgamma is not None:
        check(dgamma, wg, ref.sum_error(max(n, 1), np.abs(dy * h).sum(0)) + (np.abs(dy) * eh).sum(0), "dgamma")
    if dbeta is not None:
        check(dbeta, wb, ref.sum_error(max(n, 1), np.abs(dy).sum(0)), "dbeta")


NORM_SIZES = [(1, 1), (1, 602), (3, 2), (5, 3), (2, 7), (9, 8), (64, 16), (70, 17), (33, 33), (100, 64), (513, 100), (130, 128), (77, 255), (300, 256), (1024, 602),
              (40, 1000), (9, 1024), (10, 1025), (7, 1500), (6, 2048), (5, 2049), (3, 5000), (2, 65536), (70_001, 64)]


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,dim", NORM_SIZES)
def test_layer_norm(ctx, dtype, n, dim):
    rng = np.random.default_rng(n + dim)
    x = torch.from_numpy(rng.normal(size=(n, dim)) * 1.5 + rng.normal(size=(n, 1)) * 3).to(dtype)
    gamma, beta = torch.from_numpy(rng.normal(size=dim)).float(), torch.from_numpy(rng.normal(size=dim)).float()
    given = n % 2 == 0
    flat_x, vx = padded(x, dtype, dim % 3, n % 2)
    flat, y = padded(torch.zeros(n, dim), dtype, dim % 4, dim % 2)
    mean, rstd = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    ctx.layer_norm(vx, n, dim, gamma.to(DEV) if given else None, beta.to(DEV) if given else None, 1e-5, y, mean, rstd)
    torch.cuda.synchronize()
    check_norm(y, mean, rstd, f64(x), f64(gamma) if given else np.ones(dim), f64(beta) if given else np.zeros(dim), 1e-5, dtype)
    assert untouched(flat, y)
    if dim < 5000:                                         # in place, and without the statistics: the same bits
        want = y.clone()
        ctx.layer_norm(vx, n, dim, gamma.to(DEV) if given else None, beta.to(DEV) if given else None, 1e-5, vx)
        assert torch.equal(vx, want) and untouched(flat_x, vx)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,dim", NORM_SIZES + [(0, 30), (0, 3000)])
def test_layer_norm_gradient(ctx, dtype, n, dim):
    rng = np.random.default_rng(n + dim)
    rows = max(n, 1)
    x = torch.from_numpy(rng.normal(size=(rows, dim)) * 1.5 + rng.normal(size=(rows, 1)) * 3).to(dtype)
    dy = torch.from_numpy(rng.normal(size=(rows, dim)) * 0.1).to(dtype)
    gamma = torch.from_numpy(rng.normal(size=dim)).float() if n % 2 == 0 else None
    g64 = f64(gamma) if gamma is not None else np.ones(dim)
    x64, dy64 = f64(x)[:n], f64(dy)[:n]
    mean = torch.from_numpy(x64.mean(1)).float()
    rstd = torch.from_numpy(1.0 / np.sqrt(x64.var(1) + 1e-5)).float()
    _, vx = padded(x, dtype, dim % 3, n % 2)
    _, vdy = padded(dy, dtype, dim % 2, 0)
    flat, dx = padded(torch.zeros(rows, dim), dtype, dim % 4, dim % 2)
    dg, db = torch.full((dim,), PAD, device=DEV), torch.full((dim,), PAD, device=DEV)
    one = torch.zeros(1, device=DEV)
    args = (n, dim, gamma.to(DEV) if gamma is not None else None, mean.to(DEV) if n else one, rstd.to(DEV) if n else one)
    ctx.layer_norm_grad(vdy, vx, *args, dx, dg, db)
    torch.cuda.synchronize()
    check_norm_grad(dx[:n], dg, db, dy64, x64, g64, f64(mean), f64(rstd), dtype)
    if n:
        assert untouched(flat, dx)
    # one output at a time, and dx in dy's place: the same bits
    dg2, db2 = torch.full((dim,), PAD, device=DEV), torch.full((dim,), PAD, device=DEV)
    ctx.layer_norm_grad(vdy, vx, *args, None, dg2, None)
    ctx.layer_norm_grad(vdy, vx, *args, None, None, db2)
    assert torch.equal(dg2, dg) and torch.equal(db2, db)
    if n:
        want = dx.clone()
        ctx.layer_norm_grad(vdy, vx, *args, vdy, None, None)
        assert torch.equal(vdy, want)


def test_layer_norm_of_rows_without_spread_and_of_far_sizes(ctx):
    n, dim = 8, 100
    x = torch.zeros(n, dim)
    x[0] = 1.1                                              # no spread: what is left is the rounding of the mean
    x[1] = 1e30 * (torch.arange(dim) % 2)                   # squares that overflow 32 bits: rstd 0, as the formula in 32 bits
    x[2] = 1e-20 * torch.arange(dim)
    x[3] = 1000.0 + torch.arange(dim) / 1000.0
    x[4, 0] = float("nan")
    x[5, 9] = float("inf")
    y, mean, rstd = torch.empty(n, dim, device=DEV), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    ctx.layer_norm(x.to(DEV), n, dim, None, None, 1e-5, y, mean, rstd)
    assert bool(y[4].isnan().all() and y[5].isnan().any())
    for rows in ([0], [2], [3], [6, 7]):
        check_norm(y[rows], mean[rows], rstd[rows], f64(x)[rows], np.ones(dim), np.zeros(dim), 1e-5, F32)
    assert bool((y[6:] == 0).all() and (mean[6:] == 0).all())


def test_layer_norm_gradient_is_the_difference_quotient(ctx):
    """Along a direction: central differences of the kernel's own forward pass, whose 32-bit noise and third derivative bound the step."""
    rng = np.random.default_rng(4)
    n, dim, eps, step = 6, 50, 1e-3, 2.0 ** -7
    x, dy, way = (torch.from_numpy(rng.normal(size=(n, dim))).float() for _ in range(3))
    gamma, beta = (torch.from_numpy(rng.normal(size=dim)).float().to(DEV) for _ in range(2))
    y, mean, rstd, dx = (torch.empty(s, device=DEV) for s in ((n, dim), (n,), (n,), (n, dim)))
    ctx.layer_norm(x.to(DEV), n, dim, gamma, beta, eps, y, mean, rstd)
    ctx.layer_norm_grad(dy.to(DEV), x.to(DEV), n, dim, gamma, mean, rstd, dx, None, None)
    ends = []
    for sign in (1, -1):
        ctx.layer_norm((x + sign * step * way).to(DEV), n, dim, gamma, beta, eps, y)
        ends.append(float((f64(y) * f64(dy)).sum()))
    slope = (ends[0] - ends[1]) / (2 * step)
    forward = lambda t: float((ref.layer_norm(f64(x) + t * f64(way), f64(gamma), f64(beta), eps)[0] * f64(dy)).sum())     # noqa: E731
    exact = (forward(step) - forward(-step)) / (2 * step)                                     # the same quotient in 64 bits
    noise = 2 * 2.0 ** -24 * 40 * float(np.abs(f64(y) * f64(dy)).sum()) / (2 * step)
    assert abs(slope - exact) <= noise
    third = abs((forward(2 * step) - 2 * forward(step) + 2 * forward(-step) - forward(-2 * step)) / (2 * step ** 3))
    along = float((f64(dx) * f64(way)).sum())
    assert abs(along - slope) <= noise + third * step ** 2 / 3 + 2.0 ** -18 * float(np.abs(f64(dx) * f64(way)).sum())


# ---------------------------------------------------------------- clipping
def clip_case(rng, sizes, types, std):
    return [torch.from_numpy(rng.normal(size=k) * std).to(t) for k, t in zip(sizes, types)]


CLIP_SIZES = [[], [0], [1], [5, 0, 3], [8191, 8192, 8193], [1, 2, 3, 4, 5, 6, 7, 9, 100, 1000], [16] * 64, [17] * 65, [1] * 300 + [100_000], [3_000_001, 77],
              [4096] * 130]


@pytest.mark.parametrize("types", ["f32", "bf16", "f16", "mixed"])
@pytest.mark.parametrize("which", range(len(CLIP_SIZES)))
@pytest.mark.parametrize("share", [0.25, 2.0])
def test_clip(ctx, types, which, share):
    """The norm clipped to a quarter of itself, or left alone; into other arrays and in place."""
    from paper_2505_10806_amd import binding as B
    sizes = CLIP_SIZES[which]
    rng = np.random.default_rng(which)
    kinds = [dict(f32=F32, bf16=torch.bfloat16, f16=torch.float16).get(types, ref.TYPES[i % 3]) for i in range(len(sizes))]
    grads = clip_case(rng, sizes, kinds, 0.02)
    norm64, _ = ref.clip([f64(g) for g in grads], 1.0)
    most = float(np.float32(norm64 * share))
    _, want = ref.clip([f64(g) for g in grads], most)
    buffers = [torch.full((k + 9,), PAD, dtype=t, device=DEV) for k, t in zip(sizes, kinds)]
    out = [b[i % 8:i % 8 + k] for i, (b, k) in enumerate(zip(buffers, sizes))]               # any alignment
    there = [g.to(DEV) for g in grads]
    norm = torch.full((1,), PAD, device=DEV)
    ctx.clip_grad_norm(B.TensorList(there, out), most, norm)
    check(norm, np.array([norm64]), 2.0 ** -23 * norm64, "norm")
    ctx.clip_grad_norm(B.TensorList(there), most, norm)
    for i, (o, t, w, k, kind) in enumerate(zip(out, there, want, sizes, kinds)):
        check(o, w, 2.0 ** -22 * np.abs(w) + ref.stored(w, kind), f"tensor {i}")
        assert torch.equal(t, o)
        if share > 1:
            assert torch.equal(o.cpu(), grads[i])
        assert int((buffers[i] != PAD).sum()) <= k and bool((buffers[i][i % 8 + k:] == PAD).all())


def test_clip_what_is_not_finite_or_far(ctx):
    from paper_2505_10806_amd import binding as B
    norm = torch.zeros(1, device=DEV)
    for bad in (float("inf"), float("nan"), -float("inf")):
        g = [torch.ones(10, device=DEV), torch.tensor([1.0, bad], device=DEV)]
        out = [torch.empty_like(t) for t in g]
        ctx.clip_grad_norm(B.TensorList(g, out), 1.0, norm)
        assert not np.isfinite(norm.item()) and torch.equal(out[0], g[0]) and torch.equal(out[1].nan_to_num(), g[1].nan_to_num())
    huge = [torch.full((1000,), 3e38, device=DEV)]                                           # squares overflow 32 bits, the norm too
    out = [torch.empty_like(huge[0])]
    ctx.clip_grad_norm(B.TensorList(huge, out), 1.0, norm)
    assert norm.item() == float("inf") and np.allclose(f64(out[0]), 1000 ** -0.5, rtol=1e-6)  # (the norm itself is finite in 64 bits)
    small = [torch.full((1000,), 1e-30, device=DEV)]
    ctx.clip_grad_norm(B.TensorList(small, out), 1e-31, norm)
    assert abs(norm.item() / (1e-30 * 1000 ** 0.5) - 1) < 1e-6 and np.allclose(f64(out[0]), 1e-31 * 1000 ** -0.5, rtol=1e-5)
    ctx.clip_grad_norm(B.TensorList([torch.zeros(5, device=DEV)]), 0.0, norm)
    assert norm.item() == 0.0
    g = torch.ones(7, device=DEV)
    ctx.clip_grad_norm(B.TensorList([g]), 0.0, norm)
    assert bool((g == 0).all())
    g = torch.ones(7, device=DEV)
    ctx.clip_grad_norm(B.TensorList([g]), float("inf"), norm)
    assert bool((g == 1).all()) and abs(norm.item() - 7 ** 0.5) < 1e-6


# ---------------------------------------------------------------- large results
@pytest.mark.parametrize("dtype", ref.TYPES)
def test_results_larger_than_the_caches(ctx, dtype):
    """More than 32 MiB of results in rows of whole 16 bytes are stored another way."""
    from paper_2505_10806_amd import binding as B
    n, dim = (140_007, 64) if dtype == F32 else (270_011, 64)
    rng = np.random.default_rng(n)
    gen = torch.Generator(device=DEV).manual_seed(n)
    x = torch.randn(n, dim, generator=gen, device=DEV).to(dtype)
    some = np.concatenate([np.arange(40), rng.integers(0, n, 2000), np.arange(n - 40, n)])
    at = torch.from_numpy(some).to(DEV)
    packed, back = B.mx4_rows(n, dim, DEV), torch.empty(n, dim, dtype=dtype, device=DEV)
    ctx.mx4_quantize(x, n, dim, packed)
    ctx.mx4_dequantize(packed, n, dim, back)
    bytes_, values = ref.quantize(f64(x[at]))
    assert np.array_equal(of_packed(packed[at], dim), bytes_) and np.array_equal(f64(back[at]), f64(torch.from_numpy(values).to(dtype)))
    wb, wv = packed_rows(rng, dim, dim)
    ctx.mx4_matmul(packed, n, to_packed(wb), dim, dim, back)
    check(back[at], values @ wv.T, sum_allowed(dim, values, wv, dtype), "y")
    y, mean, rstd = torch.empty_like(x), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    ctx.layer_norm(x, n, dim, None, None, 1e-5, y, mean, rstd)
    check_norm(y[at], mean[at], rstd[at], f64(x[at]), np.ones(dim), np.zeros(dim), 1e-5, dtype)
    dy = torch.randn(n, dim, generator=gen, device=DEV).to(dtype)
    dx, dg, db = torch.empty_like(x), torch.empty(dim, device=DEV), torch.empty(dim, device=DEV)
    ctx.layer_norm_grad(dy, x, n, dim, None, mean, rstd, dx, dg, db)
    check_norm_grad(dx[at], None, None, f64(dy[at]), f64(x[at]), np.ones(dim), f64(mean[at]), f64(rstd[at]), dtype)
    check_norm_grad(None, dg, db, f64(dy), f64(x), np.ones(dim), f64(mean), f64(rstd), dtype)
    norm, out = torch.empty(1, device=DEV), torch.empty_like(dy)
    ctx.clip_grad_norm(B.TensorList([dy, dx], [out, back]), 7.0, norm)
    norm64, _ = ref.clip([f64(dy), f64(dx)], 7.0)
    check(norm, np.array([norm64]), 2.0 ** -23 * norm64, "norm")
    for g, o in ((dy, out), (dx, back)):
        want = f64(g[at]) * (7.0 / norm64)
        check(o[at], want, 2.0 ** -22 * np.abs(want) + ref.stored(want, dtype), "clipped")


# ---------------------------------------------------------------- far addresses, streams, graphs
def test_rows_beyond_32_bits(ctx):
    """Row offsets that pass 2^32 numbers, in every array."""
    n, dim, out = 65_600, 40, 33
    stride = 65_552                                       # n * stride = 4.3e9 numbers
    words = ref.words(dim)
    rng = np.random.default_rng(1)
    x = torch.from_numpy(rng.normal(size=(n, dim))).half()
    far = torch.empty(n * stride, dtype=torch.float16, device=DEV).view(n, stride)
    far[:, :dim] = x.to(DEV)
    want, values = ref.quantize(f64(x[-600:]))
    store = torch.empty(n * stride, dtype=F32, device=DEV).view(n, stride)
    ctx.mx4_quantize(far, n, dim, store)
    assert np.array_equal(of_packed(store[-600:, :words].contiguous(), dim), want)
    wb, wv = packed_rows(rng, out, dim)
    ctx.mx4_matmul(store, n, to_packed(wb), out, dim, far)
    check(far[-600:, :out], values @ wv.T, sum_allowed(dim, values, wv, torch.float16), "y")
    first = ref.quantize(f64(x[:600]))[1]
    check(far[:600, :out], first @ wv.T, sum_allowed(dim, first, wv, torch.float16), "y")
    ctx.mx4_dequantize(store, n, dim, far)
    assert np.array_equal(f64(far[-600:, :dim]), f64(torch.from_numpy(values).float().half()))
    del store
    torch.cuda.empty_cache()
    near = far[:, :dim].contiguous()
    full = ref.quantize(f64(near.float()))[0]             # (numbers that are packed numbers already)
    rows = to_packed(full)
    grad = torch.empty(out, dim, device=DEV)
    ctx.mx4_matmul_grad(far, rows, n, out, dim, grad)
    other = torch.empty(out, dim, device=DEV)
    ctx.mx4_matmul_grad(near, rows, n, out, dim, other)
    assert torch.equal(grad, other)
    mean, rstd = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    y = torch.empty(n, dim, dtype=torch.float16, device=DEV)
    ctx.layer_norm(near, n, dim, None, None, 1e-5, y, mean, rstd)
    dg = [torch.empty(dim, device=DEV) for _ in range(4)]
    dx = torch.empty(n, dim, dtype=torch.float16, device=DEV)
    ctx.layer_norm_grad(near, near, n, dim, None, mean, rstd, dx, dg[0], dg[1])
    ctx.layer_norm_grad(far, far, n, dim, None, mean, rstd, far, dg[2], dg[3])
    assert torch.equal(far[:, :dim], dx) and torch.equal(dg[0], dg[2]) and torch.equal(dg[1], dg[3])
    far[:, :dim] = near
    ctx.layer_norm(far, n, dim, None, None, 1e-5, far)
    assert torch.equal(far[:, :dim], y)


def _step(ctx, B, s, stream=None):
    """One pass through every operator on the buffers of `s`."""
    n, dim, out = s["n"], s["dim"], s["out"]
    ctx.mx4_quantize(s["x"], n, dim, s["rows"], stream=stream)
    ctx.mx4_quantize(s["w"], out, dim, s["weight"], stream=stream)
    ctx.mx4_matmul(s["rows"], n, s["weight"], out, dim, s["y"], stream=stream)
    ctx.layer_norm(s["y"], n, out, s["gamma"], s["beta"], 1e-5, s["z"], s["mean"], s["rstd"], stream=stream)
    ctx.layer_norm_grad(s["z"], s["y"], n, out, s["gamma"], s["mean"], s["rstd"], s["dy"], s["dgamma"], s["dbeta"], stream=stream)
    ctx.mx4_matmul_grad(s["dy"], s["rows"], n, out, dim, s["dw"], stream=stream)
    ctx.clip_grad_norm(s["list"], 0.5, s["norm"], stream=stream)


def _buffers(B, n, dim, out, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=gen, device=DEV)                      # noqa: E731
    s = dict(n=n, dim=dim, out=out, x=rand(n, dim), w=rand(out, dim), gamma=rand(out), beta=rand(out))
    s.update(rows=B.mx4_rows(n, dim, DEV), weight=B.mx4_rows(out, dim, DEV))
    s.update({k: torch.zeros(n, out, device=DEV) for k in ("y", "z", "dy")}, mean=torch.zeros(n, device=DEV), rstd=torch.zeros(n, device=DEV),
             dgamma=torch.zeros(out, device=DEV), dbeta=torch.zeros(out, device=DEV), dw=torch.zeros(out, dim, device=DEV), norm=torch.zeros(1, device=DEV))
    s["clipped"] = [torch.zeros_like(s[k]) for k in ("dw", "dgamma", "dbeta")]
    s["list"] = B.TensorList([s["dw"], s["dgamma"], s["dbeta"]], s["clipped"])
    return s


_RESULTS = ("rows", "weight", "y", "z", "mean", "rstd", "dy", "dgamma", "dbeta", "dw", "norm")


@pytest.mark.parametrize("n", [100, 20_000])
def test_a_step_replays_from_a_hip_graph_and_repeats_bit_for_bit(ctx, n):
    from paper_2505_10806_amd import binding as B
    s, e = _buffers(B, n, 100, 128, 1), _buffers(B, n, 100, 128, 1)
    _step(ctx, B, s)                                       # grows the scratch
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph.capture_begin(capture_error_mode="relaxed")
        _step(ctx, B, s)
        graph.capture_end()
    torch.cuda.synchronize()
    for replay in range(3):
        x = torch.randn(n, 100, generator=torch.Generator(device=DEV).manual_seed(50 + replay), device=DEV)
        e["x"].copy_(x)
        _step(ctx, B, e)                                   # eager work between the replays, on the same scratch
        torch.cuda.synchronize()
        for k in _RESULTS:
            s[k].fill_(PAD)
            if k in ("rows", "weight"):                    # (what lies behind a row is never written)
                words = B.mx4_row_words(100)
                s[k][:, words:] = e[k][:, words:]
        s["x"].copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        for k in _RESULTS:
            assert torch.equal(s[k].view(torch.int32), e[k].view(torch.int32)), (replay, k)
        for a, b in zip(s["clipped"], e["clipped"]):
            assert torch.equal(a, b)
    del graph


def test_a_step_on_another_stream(ctx):
    from paper_2505_10806_amd import binding as B
    s, e = _buffers(B, 5000, 64, 47, 2), _buffers(B, 5000, 64, 47, 2)
    _step(ctx, B, e)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    _step(ctx, B, s, stream=side)
    side.synchronize()
    for k in _RESULTS:
        assert torch.equal(s[k].view(torch.int32), e[k].view(torch.int32)), k


def test_packed_rows_go_through_the_gather_as_they_are(ctx):
    """Packed stores (the remote one in pinned memory, packed there), a cache of packed rows, a gather: the batch's packed rows, bit for bit."""
    from paper_2505_10806_amd import binding as B
    nodes, dim, capacity = 3000, 100, 500
    rng = np.random.default_rng(12)
    x = torch.from_numpy(rng.normal(size=(nodes, dim))).float()
    words = B.mx4_row_words(dim)
    owner = np.arange(nodes) % 2                            # every other node is remote
    rank = np.arange(nodes) // 2
    home = torch.from_numpy((np.where(owner == 0, 0, 2) << 30 | rank).astype(np.uint32).view(np.int32)).to(DEV)
    local, remote = B.mx4_rows(nodes // 2, dim, DEV), B.mx4_rows(nodes // 2, dim, "cpu", pin_memory=True)
    ctx.mx4_quantize(x[0::2].contiguous().to(DEV), nodes // 2, dim, local)
    ctx.mx4_quantize(x[1::2].contiguous().pin_memory(), nodes // 2, dim, remote)
    torch.cuda.synchronize()
    want = ref.quantize(f64(x))[0]
    assert np.array_equal(of_packed(remote, dim), want[1::2])
    counts = torch.from_numpy(rng.integers(1, 50, size=nodes).astype(np.int32)).to(DEV)
    cache = B.FeatureCache(nodes, capacity, local.shape[1], DEV)
    ctx.build_cache(counts, home, remote, words, cache)
    ids = torch.from_numpy(rng.permutation(nodes)[:1777].astype(np.int32)).to(DEV)
    out, stats = B.mx4_rows(1777, dim, DEV), torch.zeros(3, dtype=torch.int64, device=DEV)
    ctx.gather_features(ids, 1777, cache, local, remote, words, out, stats)
    torch.cuda.synchronize()
    assert np.array_equal(of_packed(out, dim), want[ids.cpu().numpy()]) and int(stats[1]) > 0 and int(stats[2]) > 0
