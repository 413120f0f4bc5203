"""Softmax cross entropy and its gradients on an MI355X against their 64-bit forms (tests/vector_reference.py).

Tolerances: z errs by a 32-bit sum of dim products (sum_error); 32-bit numbers are cut to parts of 8 bits, which leaves up to 2^-7 and 2^-15 of a
number for the second and third, and the three products of parts that are left out are below 2 * 2^-22 + 2^-30 < 2^-20 of the product.  exp and log go through
base 2, which rounds z / ln 2 and lse / ln 2 (2^-24 of each, twice); the hardware's exp2 and log2 err by an ulp or two, 2^-22.  An error d of z is one of p d in p.
Sums of p over the classes and of g over rows or classes are 32-bit sums.  For its products g is rounded to the rows' type (for f16 after a factor 2^14, so its
smallest step is 2^-38), f32 cut as above."""
import numpy as np
import pytest
import torch

import training_reference as ref
import vector_reference as vec
from test_gpu_training_ops import DEV, F32, PAD, check, ctx, f64, padded, untouched, _name_the_case  # noqa: F401  (fixtures among them)

pytestmark = pytest.mark.gpu
CUT = 2.0 ** -20
# (and where one kernel hands over to the next: 8 numbers, 128, 256, 512; 32 rows; 64 classes)
SIZES = [(32, 65, 8), (33, 64, 512), (32, 300, 7), (64, 64, 256), (65, 66, 257), (2000, 64, 513), (31, 9000, 130), (32, 700, 640), (500, 33, 384), (257, 65, 8), (400, 2, 513), (1, 1, 1), (1, 2, 3), (2, 31, 7), (3, 64, 8), (31, 33, 9), (33, 41, 16), (64, 47, 17), (65, 65, 64), (63, 63, 100), (100, 257, 100), (129, 1000, 127),
         (256, 128, 128), (257, 300, 129), (300, 70, 256), (5, 4097, 300), (200, 41, 602), (70, 130, 1025), (1000, 47, 33), (3000, 10, 40), (1, 20_000, 100), (40, 3, 3000)]


def inputs(rng, n, classes, dim, dtype, extra=0, offset=0, spread=2.0):
    fx, x = padded(rng.normal(size=(n, dim)), dtype, extra, offset)
    fw, w = padded(rng.normal(size=(classes, dim)) * spread * dim ** -0.5, dtype, extra, offset)
    labels = rng.integers(0, classes, size=n)
    strange = np.array([-1, classes, 2 ** 31 - 1, -2 ** 31])
    if n > 2:
        labels = np.where(rng.random(n) < 0.1, strange[rng.integers(0, 4, n)], labels)
    return x, w, labels


def on_gpu(ids):
    return torch.from_numpy(ids.astype(np.int32)).to(DEV)


def z_error(x, w, dtype):
    size = np.abs(x) @ np.abs(w).T
    return ref.sum_error(x.shape[1], size) + (CUT * size if dtype == F32 else 0.0)


def check_loss(loss, lse, x, w, labels, dtype, what=""):
    z = vec.logits(x, w)
    want, want_lse = vec.cross_entropy(z, labels)
    ez = z_error(x, w, dtype).max(1)
    counts = (labels >= 0) & (labels < len(w))
    allowed = ez + 2.0 ** -22 * (np.abs(z).max(1) + np.abs(want_lse) + 2.0) + ref.sum_error(len(w), 1.0)
    check(lse, want_lse, np.where(counts, allowed, 0.0), "lse" + what)
    check(loss, want, np.where(counts, allowed + ez + 2.0 ** -23 * np.abs(want), 0.0), "loss" + what)


def check_grads(dx, dw, x, w, labels, lse, share, dtype, what=""):
    z = vec.logits(x, w)
    want_dx, want_dw, p, g = vec.cross_entropy_grad(z, labels, lse, share, x, w)
    counts = (labels >= 0) & (labels < len(w))
    share = np.where(counts, np.abs(share), 0.0)[:, None]
    eg = share * p * (z_error(x, w, dtype) + 2.0 ** -22 * (np.abs(z) + np.abs(lse)[:, None] + 2.0))
    eg += np.abs(g) * (2.0 ** -23 + (CUT if dtype == F32 else ref.HALF_ULP[dtype]))
    # (f16's smallest step times the largest share; for dx the row's own)
    step = 2.0 ** -38 if dtype == torch.float16 else 0.0
    if dx is not None:
        allowed = eg @ np.abs(w) + ref.sum_error(len(w), np.abs(g) @ np.abs(w)) + step * share * np.abs(w).sum(0)
        check(dx, want_dx, np.where(counts[:, None], allowed + ref.stored(want_dx, dtype), 0.0), "dx" + what)
    if dw is not None:
        allowed = eg.T @ np.abs(x) + ref.sum_error(len(x), np.abs(g).T @ np.abs(x)) + step * share.max(initial=0.0) * np.abs(x * counts[:, None]).sum(0)
        check(dw, want_dw, allowed + ref.stored(want_dw, dtype), "dweight" + what)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,classes,dim", SIZES)
def test_loss(ctx, dtype, n, classes, dim):  # noqa: F811
    rng = np.random.default_rng(n + classes + dim)
    x, w, labels = inputs(rng, n, classes, dim, dtype)
    loss, lse = torch.full((n + 1,), PAD, device=DEV), torch.full((n + 1,), PAD, device=DEV)
    ctx.cross_entropy(x, n, dim, w, classes, on_gpu(labels), loss, lse)
    check_loss(loss[:n], lse[:n], f64(x), f64(w), labels, dtype)
    assert float(loss[n]) == PAD and float(lse[n]) == PAD


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,classes,dim", SIZES)
def test_gradients(ctx, dtype, n, classes, dim):  # noqa: F811
    rng = np.random.default_rng(n + classes + dim + 1)
    x, w, labels = inputs(rng, n, classes, dim, dtype)
    _, lse64 = vec.cross_entropy(vec.logits(f64(x), f64(w)), labels)
    lse = torch.from_numpy(lse64).float().to(DEV)
    for weights in (False, True):
        dloss = torch.from_numpy(rng.random(n) * 3.0).float().to(DEV) if weights else None
        scale = 0.75
        fx, dx = padded(torch.zeros(n, dim), dtype)
        fw, dw = padded(torch.zeros(classes, dim), dtype)
        ctx.cross_entropy_grad(x, n, dim, w, classes, on_gpu(labels), lse, dx, dw, dloss=dloss, scale=scale)
        share = np.full(n, scale) if dloss is None else f64(dloss) * scale
        check_grads(dx, dw, f64(x), f64(w), labels, f64(lse), share, dtype)
        assert untouched(fx, dx) and untouched(fw, dw)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,classes,dim,extra,offset", [(70, 90, 100, 1, 1), (70, 90, 64, 7, 3), (5, 5, 7, 5, 2), (300, 30, 130, 3, 1)])
def test_strides_and_alignment(ctx, dtype, n, classes, dim, extra, offset):  # noqa: F811
    """What lies behind the rows' numbers is neither read (NaN there would show) nor written."""
    rng = np.random.default_rng(n)
    x, w, labels = inputs(rng, n, classes, dim, dtype, extra, offset)
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    for t, rows in ((x, n), (w, classes)):
        torch.as_strided(t, (rows, dim + extra), t.stride(), t.storage_offset())[:, dim:] = float("nan")
    ctx.cross_entropy(x, n, dim, w, classes, on_gpu(labels), loss, lse)
    check_loss(loss, lse, f64(x), f64(w), labels, dtype)
    fx, dx = padded(torch.zeros(n, dim), dtype, extra, offset)
    fw, dw = padded(torch.zeros(classes, dim), dtype, extra, offset)
    ctx.cross_entropy_grad(x, n, dim, w, classes, on_gpu(labels), lse, dx, dw)
    check_grads(dx, dw, f64(x), f64(w), labels, f64(lse), np.ones(n), dtype)
    assert untouched(fx, dx) and untouched(fw, dw)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,classes,dim", [(200, 60, 70), (200, 100, 70), (30, 100, 70), (200, 100, 200), (200, 100, 300), (200, 64, 300)])
def test_rows_that_do_not_count_may_hold_anything(ctx, dtype, n, classes, dim):  # noqa: F811
    rng = np.random.default_rng(4)
    x, w, labels = inputs(rng, n, classes, dim, dtype)
    gone = ~((labels >= 0) & (labels < classes))
    at = torch.from_numpy(np.flatnonzero(gone)).to(DEV)
    clean = f64(x)
    x[at] = float("nan")
    x[at[0]] = float("inf")
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    ctx.cross_entropy(x, n, dim, w, classes, on_gpu(labels), loss, lse)
    check_loss(loss, lse, clean, f64(w), labels, dtype)
    lse64 = f64(lse)
    lse[at] = float("nan")
    dloss = torch.ones(n, device=DEV)
    dloss[at] = float("-inf")
    dx, dw = torch.full((n, dim), PAD, dtype=dtype, device=DEV), torch.full((classes, dim), PAD, dtype=dtype, device=DEV)
    ctx.cross_entropy_grad(x, n, dim, w, classes, on_gpu(labels), lse, dx, dw, dloss=dloss)
    check_grads(dx, dw, clean, f64(w), labels, lse64, np.ones(n), dtype)
    # none counts: zeros, even of a weight that is not finite
    w[3] = float("inf")
    w[4, 2] = float("nan")
    nobody = on_gpu(np.full(n, -1))
    ctx.cross_entropy(x, n, dim, w, classes, nobody, loss, lse)
    assert bool((loss == 0).all()) and bool((lse == 0).all())
    ctx.cross_entropy_grad(x, n, dim, w, classes, nobody, lse, dx, dw)
    assert bool((dx == 0).all()) and bool((dw == 0).all())


@pytest.mark.parametrize("n,classes,dim", [(100, 70, 90), (100, 41, 90), (100, 64, 300), (20, 700, 90), (100, 70, 300), (100, 90, 200)])
@pytest.mark.parametrize("live", [0, 1, 64, 100, 101, -2])
def test_counts_on_the_device(ctx, live, n, classes, dim):  # noqa: F811
    rng = np.random.default_rng(live + 20)
    real = max(0, min(n, live))
    n_dev = torch.tensor([live], dtype=torch.int32, device=DEV)
    for dtype in ref.TYPES:
        x, w, labels = inputs(rng, n, classes, dim, dtype)
        x[real:] = float("nan")
        loss, lse = torch.full((n,), PAD, device=DEV), torch.full((n,), PAD, device=DEV)
        ctx.cross_entropy(x, n, dim, w, classes, on_gpu(labels), loss, lse, n_dev=n_dev)
        assert bool((loss[real:] == PAD).all() and (lse[real:] == PAD).all())
        dx, dw = torch.full((n, dim), PAD, dtype=dtype, device=DEV), torch.full((classes, dim), PAD, dtype=dtype, device=DEV)
        saved = lse.clone()
        saved[real:] = float("nan")
        ctx.cross_entropy_grad(x, n, dim, w, classes, on_gpu(labels), saved, dx, dw, n_dev=n_dev)
        assert bool((dx[real:] == PAD).all())
        if real == 0:
            assert bool((dw == 0).all())
            continue
        check_loss(loss[:real], lse[:real], f64(x)[:real], f64(w), labels[:real], dtype)
        check_grads(dx[:real], dw, f64(x)[:real], f64(w), labels[:real], f64(lse)[:real], np.ones(real), dtype)


def test_outputs_that_are_not_wanted(ctx):  # noqa: F811
    rng = np.random.default_rng(5)
    n, classes, dim = 90, 33, 50
    x, w, labels = inputs(rng, n, classes, dim, F32)
    both = [torch.empty(n, device=DEV) for _ in range(2)]
    ctx.cross_entropy(x, n, dim, w, classes, on_gpu(labels), *both)
    one = torch.empty(n, device=DEV)
    ctx.cross_entropy(x, n, dim, w, classes, on_gpu(labels), one, None)
    assert torch.equal(one, both[0])
    ctx.cross_entropy(x, n, dim, w, classes, on_gpu(labels), None, one)
    assert torch.equal(one, both[1])
    dx, dw = torch.empty(n, dim, device=DEV), torch.empty(classes, dim, device=DEV)
    ctx.cross_entropy_grad(x, n, dim, w, classes, on_gpu(labels), one, dx, dw)
    alone = torch.empty_like(dx), torch.empty_like(dw)
    ctx.cross_entropy_grad(x, n, dim, w, classes, on_gpu(labels), one, alone[0], None)
    ctx.cross_entropy_grad(x, n, dim, w, classes, on_gpu(labels), one, None, alone[1])
    assert torch.equal(dx, alone[0]) and torch.equal(dw, alone[1])
    ctx.cross_entropy_grad(x, 0, dim, w, classes, on_gpu(labels), one, None, dw)
    assert bool((dw == 0).all())


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,classes,dim", [(64, 100, 40), (64, 60, 40), (64, 2000, 40), (64, 400, 200), (64, 400, 300)])
def test_large_and_small_logits(ctx, dtype, n, classes, dim):  # noqa: F811
    """Rows far from zero, a class that takes everything, all classes alike, and lse far below zero."""
    rng = np.random.default_rng(6)
    x, w, labels = inputs(rng, n, classes, dim, dtype)
    x[:16] *= 60.0
    x[16:20] = 0.0
    w[:, 0] = -20.0 * torch.rand(classes, device=DEV).to(dtype) - 10.0
    x[20:40, 0] = 30.0
    w[7] = w[8]
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    ctx.cross_entropy(x, n, dim, w, classes, on_gpu(labels), loss, lse)
    check_loss(loss, lse, f64(x), f64(w), labels, dtype)
    assert float(lse[20:40].min()) < -100.0
    dx, dw = torch.empty(n, dim, dtype=dtype, device=DEV), torch.empty(classes, dim, dtype=dtype, device=DEV)
    ctx.cross_entropy_grad(x, n, dim, w, classes, on_gpu(labels), lse, dx, dw)
    check_grads(dx, dw, f64(x), f64(w), labels, f64(lse), np.ones(n), dtype)


def test_a_class_that_is_shut_out(ctx):  # noqa: F811
    """16-bit rows whose first number is 1 shut a class out by a weight of -infinity there: it has probability 0 and no gradient but NaN's absence."""
    rng = np.random.default_rng(7)
    n, classes, dim = 80, 70, 24
    x, w, labels = inputs(rng, n, classes, dim, torch.bfloat16)
    x[:, 0] = 1.0
    labels = np.where(labels == 5, 6, labels)
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    w[5, 0] = float("-inf")
    ctx.cross_entropy(x, n, dim, w, classes, on_gpu(labels), loss, lse)
    rest = np.delete(np.arange(classes), 5)
    moved = np.where(labels > 5, labels - 1, labels)
    moved = np.where((labels >= 0) & (labels < classes), moved, -1)
    check_loss(loss, lse, f64(x), f64(w)[rest], moved, torch.bfloat16)
    dw = torch.empty(classes, dim, dtype=torch.bfloat16, device=DEV)
    ctx.cross_entropy_grad(x, n, dim, w, classes, on_gpu(labels), lse, None, dw)
    assert bool((dw[5] == 0).all())
    check_grads(None, dw[torch.from_numpy(rest).to(DEV)], f64(x), f64(w)[rest], moved, f64(lse), np.ones(n), torch.bfloat16)


def test_not_a_number_stays_in_its_row(ctx):  # noqa: F811
    rng = np.random.default_rng(9)
    n, classes, dim = 70, 80, 30
    for dtype in ref.TYPES:
        x, w, labels = inputs(rng, n, classes, dim, dtype)
        labels = np.clip(labels, 0, classes - 1)
        x[11, 3] = float("nan")
        loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        ctx.cross_entropy(x, n, dim, w, classes, on_gpu(labels), loss, lse)
        bad = torch.isnan(loss)
        assert bool(bad[11]) and int(bad.sum()) == 1 and int(torch.isnan(lse).sum()) == 1
        dx, dw = torch.empty(n, dim, dtype=dtype, device=DEV), torch.empty(classes, dim, dtype=dtype, device=DEV)
        ctx.cross_entropy_grad(x, n, dim, w, classes, on_gpu(labels), lse, dx, dw)
        bad = torch.isnan(dx).any(1)
        assert bool(bad[11]) and int(bad.sum()) == 1 and bool(torch.isnan(dw).all())


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,classes,dim", [(700, 3000, 100), (5000, 47, 100), (20, 30_000, 100), (300, 3000, 600)])
def test_the_same_call_gives_the_same_bits(ctx, dtype, n, classes, dim):  # noqa: F811
    rng = np.random.default_rng(10)
    x, w, labels = inputs(rng, n, classes, dim, dtype)
    runs = []
    for _ in range(2):
        loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        dx, dw = torch.empty(n, dim, dtype=dtype, device=DEV), torch.empty(classes, dim, dtype=dtype, device=DEV)
        ctx.cross_entropy(x, n, dim, w, classes, on_gpu(labels), loss, lse)
        ctx.cross_entropy_grad(x, n, dim, w, classes, on_gpu(labels), lse, dx, dw)
        runs.append((loss, lse, dx, dw))
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_gradients_against_differences(ctx):  # noqa: F811
    """The gradient along a direction against the loss on both sides: (f(+h) - f(-h)) / 2h errs by h^2 / 6 of a third derivative below 60 (three directions'
    worth of z' up to 4 each) and by the losses' own 2^-21 * 64 / h."""
    rng = np.random.default_rng(12)
    n, classes, dim = 50, 37, 28
    x, w, labels = inputs(rng, n, classes, dim, F32)
    at, h = on_gpu(labels), 2.0 ** -7
    ux, uw = (torch.from_numpy(rng.normal(size=s) * dim ** -0.5).float().to(DEV) for s in ((n, dim), (classes, dim)))
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)

    def f(t):
        ctx.cross_entropy((x + t * ux).contiguous(), n, dim, (w + t * uw).contiguous(), classes, at, loss, None)
        return float(loss.double().sum())
    ctx.cross_entropy(x, n, dim, w, classes, at, None, lse)
    dx, dw = torch.empty(n, dim, device=DEV), torch.empty(classes, dim, device=DEV)
    ctx.cross_entropy_grad(x, n, dim, w, classes, at, lse, dx, dw)
    along = float((dx.double() * ux.double()).sum() + (dw.double() * uw.double()).sum())
    allowed = n * (h * h / 6.0 * 60.0 + 2.0 ** -21 * 64 / h)
    assert abs((f(h) - f(-h)) / (2 * h) - along) <= allowed


def test_recorded_into_a_graph(ctx):  # noqa: F811
    rng = np.random.default_rng(13)
    n, classes, dim = 300, 500, 60
    side = torch.cuda.Stream()
    x, w = torch.zeros(n, dim, device=DEV), torch.zeros(classes, dim, device=DEV)
    labels = torch.zeros(n, dtype=torch.int32, device=DEV)
    outs = [torch.zeros(n, device=DEV), torch.zeros(n, device=DEV), torch.zeros(n, dim, device=DEV), torch.zeros(classes, dim, device=DEV)]

    def calls(loss, lse, dx, dw, stream):
        ctx.cross_entropy(x, n, dim, w, classes, labels, loss, lse, stream=stream)
        ctx.cross_entropy_grad(x, n, dim, w, classes, labels, lse, dx, dw, scale=1.0 / n, stream=stream)
    with torch.cuda.stream(side):
        calls(*outs, side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls(*outs, torch.cuda.current_stream())
    for _ in range(3):
        x.copy_(torch.from_numpy(rng.normal(size=(n, dim))))
        w.copy_(torch.from_numpy(rng.normal(size=(classes, dim))))
        labels.copy_(on_gpu(rng.integers(-20, classes, size=n)))
        graph.replay()
        torch.cuda.synchronize()
        eager = [torch.zeros_like(t) for t in outs]
        calls(*eager, None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager))


@pytest.mark.parametrize("dtype", [torch.bfloat16, F32])
def test_weight_in_several_pieces_and_many_splits(ctx, dtype):  # noqa: F811
    """Whole numbers, whose logits are exact: rows equal to one class's weight times 8, far above all others; the loss is 0 and so are the gradients but for
    rows that are told another class."""
    n, classes, dim = 300, 1_300_000, 64
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)
    w = (torch.randint(0, 2, (classes, dim), generator=gen, device=DEV) * 2 - 1).to(dtype)
    pick = torch.randint(0, classes, (n,), generator=gen, device=DEV)
    pick[:3] = torch.tensor([0, classes - 1, 1_048_576], device=DEV)
    x = (w[pick] * 16).to(dtype)
    told = pick.clone()
    told[10:20] = (pick[10:20] + classes // 2) % classes
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    ctx.cross_entropy(x, n, dim, w, classes, told.int(), loss, lse)
    # (64 numbers of +-1: the next class agrees in 63 at most, 32 below; some rows have twins)
    z = torch.cat([x.float() @ w[i:i + 100_000].float().t() for i in range(0, classes, 100_000)], 1)
    want = torch.logsumexp(z.double(), 1)
    assert float((lse.double() - want).abs().max()) <= 2.0 ** -20 * 1024 and float((loss.double() - (want - z.gather(1, told[:, None])[:, 0].double())).abs().max()) <= 2.0 ** -20 * 1024
    dx, dw = torch.empty(n, dim, dtype=dtype, device=DEV), torch.full((classes, dim), PAD, dtype=dtype, device=DEV)
    ctx.cross_entropy_grad(x, n, dim, w, classes, told.int(), lse, dx, dw)
    g = (z.double() - lse.double()[:, None]).exp_()
    g[torch.arange(n, device=DEV), told] -= 1.0
    for got, want, size in ((dx, g @ w.double(), 64.0), (dw, g.t().contiguous() @ x.double(), 16.0 * n)):
        assert float((got.double() - want).abs().max()) <= (2.0 ** -7 if dtype != F32 else 2.0 ** -12) * size


@pytest.mark.parametrize("n,classes,dim", [(40, 200, 60), (40, 50, 60), (3, 200, 60)])
def test_shares_of_any_sign_and_size(ctx, n, classes, dim):  # noqa: F811
    """Negative shares, zeros, and shares of very different size; a share that is not a number shows in its row and in all of dweight."""
    rng = np.random.default_rng(14)
    for dtype in ref.TYPES:
        x, w, labels = inputs(rng, n, classes, dim, dtype)
        labels = np.clip(labels, 0, classes - 1)
        _, lse64 = vec.cross_entropy(vec.logits(f64(x), f64(w)), labels)
        lse = torch.from_numpy(lse64).float().to(DEV)
        dloss = torch.from_numpy(rng.normal(size=n)).float().to(DEV)
        dloss[0] = 0.0
        dloss[1] *= 2.0 ** -6
        dx, dw = torch.empty(n, dim, dtype=dtype, device=DEV), torch.empty(classes, dim, dtype=dtype, device=DEV)
        ctx.cross_entropy_grad(x, n, dim, w, classes, on_gpu(labels), lse, dx, dw, dloss=dloss, scale=-0.5)
        check_grads(dx, dw, f64(x), f64(w), labels, f64(lse), f64(dloss) * -0.5, dtype)
        dloss[2] = float("nan")
        ctx.cross_entropy_grad(x, n, dim, w, classes, on_gpu(labels), lse, dx, dw, dloss=dloss)
        bad = torch.isnan(dx).any(1)
        assert bool(bad[2]) and int(bad.sum()) == 1 and bool(torch.isnan(dw).all())


def test_two_contexts_on_two_streams(ctx):  # noqa: F811
    """Scratch belongs to a context: calls of two of them run side by side."""
    from paper_2505_10806_amd import binding as B
    rng = np.random.default_rng(15)
    other = B.Context(0)
    n, classes, dim = 600, 5000, 100
    x, w, labels = inputs(rng, n, classes, dim, torch.bfloat16)
    at = on_gpu(labels)
    lse = torch.empty(n, device=DEV)
    ctx.cross_entropy(x, n, dim, w, classes, at, None, lse)
    want = [torch.empty_like(x), torch.empty_like(w)]
    ctx.cross_entropy_grad(x, n, dim, w, classes, at, lse, *want)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for _ in range(3):
        for c, s in zip((ctx, other), streams):
            out = [torch.empty_like(x), torch.empty_like(w)]
            torch.cuda.synchronize() if len(got) < 2 else None
            c.cross_entropy_grad(x, n, dim, w, classes, at, lse, *out, stream=s)
            got.append(out)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for out in got for a, b in zip(out, want))
    other.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, F32])
def test_more_rows_or_classes_than_are_owned_at_a_time(ctx, dtype):  # noqa: F811
    """Around the lines between pieces of 2^22 owned rows and at the ends, rows of one side against few of the other; PAD behind the last."""
    many, few, dim = (1 << 22) + 300, 70, 8
    some = np.unique(np.concatenate([np.arange(80), (1 << 22) + np.arange(-80, 80), many // 2 + np.arange(40), many - 1 - np.arange(80)]))
    at = torch.from_numpy(some).to(DEV)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(11)
    rows = torch.randn(many, dim, generator=gen, device=DEV).to(dtype)
    other = torch.randn(few, dim, generator=gen, device=DEV).to(dtype)
    # many rows
    labels = torch.randint(-1, few, (many,), generator=gen, device=DEV).int()
    loss, lse = torch.full((many + 1,), PAD, device=DEV), torch.full((many + 1,), PAD, device=DEV)
    ctx.cross_entropy(rows, many, dim, other, few, labels, loss, lse)
    x, w, told = f64(rows[at]), f64(other), labels[at].long().cpu().numpy()
    check_loss(loss[at], lse[at], x, w, told, dtype)
    dx = torch.full((many + 1, dim), PAD, dtype=dtype, device=DEV)
    ctx.cross_entropy_grad(rows, many, dim, other, few, labels, lse, dx[:many], None)
    check_grads(dx[at], None, x, w, told, f64(lse[at]), np.ones(len(some)), dtype)
    assert float(loss[many]) == PAD and float(lse[many]) == PAD and bool((dx[many] == PAD).all())
    # many classes, the labels among those that are looked at
    told = np.random.default_rng(5).integers(0, len(some), few)
    labels = at[torch.from_numpy(told).to(DEV)].int()
    lse = torch.full((few,), 15.0, device=DEV)
    dw = torch.full((many + 1, dim), PAD, dtype=dtype, device=DEV)
    ctx.cross_entropy_grad(other, few, dim, rows, many, labels, lse, None, dw[:many])
    check_grads(None, dw[at], w, x, told, f64(lse), np.ones(few), dtype)
    assert bool((dw[many] == PAD).all())
