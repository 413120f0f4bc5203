"""Lookup of learned vectors and its gradient on an MI355X against their 64-bit forms (tests/vector_reference.py)."""
import numpy as np
import pytest
import torch

import training_reference as ref
import vector_reference as vec
from test_gpu_training_ops import DEV, F32, PAD, check, ctx, f64, padded, untouched, _name_the_case  # noqa: F401  (fixtures among them)

pytestmark = pytest.mark.gpu


def some_ids(rng, n, rows, pad=0.1):
    """Hubs often, some ids not in the table."""
    ids = (rng.random(n) ** 3 * rows).astype(np.int64)
    strange = np.array([-1, rows, 2 ** 31 - 1, -2 ** 31])
    return np.where(rng.random(n) < pad, strange[rng.integers(0, 4, n)], ids)


def on_gpu(ids):
    return torch.from_numpy(ids.astype(np.int32)).to(DEV)


# ---------------------------------------------------------------- lookup
@pytest.mark.parametrize("out", ref.TYPES)
@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,rows,dim,extra,offset", [(1, 1, 1, 0, 0), (1, 5, 64, 0, 0), (7, 3, 7, 2, 1), (130, 50, 8, 0, 0), (33, 9, 9, 1, 3), (1000, 300, 100, 0, 1),
                                                     (65, 400, 602, 0, 0), (40, 20, 1025, 3, 0), (3, 2, 65_533, 0, 1), (2049, 47, 256, 8, 0)])
def test_lookup(ctx, dtype, out, n, rows, dim, extra, offset):  # noqa: F811
    """A product that is rounded to 32 bits (2^-24 of it; the compiler may leave that rounding out) and stored: to 32 bits the same numbers as torch's."""
    rng = np.random.default_rng(n + dim)
    _, table = padded(rng.normal(size=(rows, dim)), dtype, extra, offset)
    flat, y = padded(torch.zeros(n, dim), out, extra, offset)
    y.fill_(PAD)
    ids = some_ids(rng, n, rows)
    scale = 16.0 if dim % 2 else 1.37
    ctx.embedding(table, rows, on_gpu(ids), n, dim, y, scale=scale)
    want = vec.embedding(f64(table), ids, float(np.float32(scale)))
    if out == F32:
        assert np.array_equal(f64(y), want.astype(np.float32))
    check(y, want, 2.0 ** -24 * np.abs(want) + ref.stored(want, out), "y")
    assert untouched(flat, y)


def test_lookup_of_padding_reads_zeros_whatever_the_table_holds(ctx):  # noqa: F811
    table = torch.full((4, 20), float("nan"), device=DEV)
    table[1], table[2] = float("inf"), -2.5
    y = torch.full((5, 20), PAD, device=DEV)
    ctx.embedding(table, 4, on_gpu(np.array([-1, 1, 4, 2, 0])), 5, 20, y, scale=2.0)
    got = f64(y)
    assert (got[0] == 0).all() and np.isposinf(got[1]).all() and (got[2] == 0).all() and (got[3] == -5.0).all() and np.isnan(got[4]).all()


@pytest.mark.parametrize("live", [0, 1, 33, 50, 51, -3])
def test_lookup_and_gradients_count_on_the_device(ctx, live):  # noqa: F811
    rng = np.random.default_rng(live + 10)
    n, rows, dim = 50, 12, 70
    real = max(0, min(n, live))
    n_dev = torch.tensor([live], dtype=torch.int32, device=DEV)
    ids = some_ids(rng, n, rows)
    table = torch.from_numpy(rng.normal(size=(rows, dim))).float().to(DEV)
    y = torch.full((n, dim), PAD, device=DEV)
    ctx.embedding(table, rows, on_gpu(ids), n, dim, y, n_dev=n_dev)
    assert np.array_equal(f64(y)[:real], vec.embedding(f64(table), ids[:real], 1.0)) and bool((y[real:] == PAD).all())
    dy = torch.from_numpy(rng.normal(size=(n, dim))).float()
    dy[real:] = float("nan")
    grad = torch.full((rows, dim), PAD, device=DEV)
    ctx.embedding_grad(dy.to(DEV), on_gpu(ids), n, dim, rows, grad, n_dev=n_dev)
    want, size, count = vec.embedding_grad(f64(dy)[:real], ids[:real], rows, 1.0)
    check(grad, want, ref.sum_error(count[:, None], size), "grad")
    few, touched, met = torch.full((rows, dim), PAD, device=DEV), torch.full((rows,), -5, dtype=torch.int32, device=DEV), torch.full((1,), -5, dtype=torch.int32, device=DEV)
    ctx.embedding_grad_rows(dy.to(DEV), on_gpu(ids), n, dim, rows, few, touched, met, n_dev=n_dev)
    check_rows(few, touched, met, want, size, count)


# ---------------------------------------------------------------- gradient
def check_rows(grad, touched, met, want, size, count):
    named = np.flatnonzero(count)
    assert int(met) == len(named)
    assert np.array_equal(touched.cpu().numpy()[:len(named)], named) and bool((touched[len(named):] == -5).all())
    check(grad[:len(named)], want[named], ref.sum_error(count[named][:, None], size[named]), "rows met")
    assert bool((grad[len(named):] == PAD).all())


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,rows,dim,extra", [(1, 1, 1, 0), (2, 100_000, 3, 1), (17, 1, 8, 0), (300, 7, 100, 0), (1000, 47, 64, 0), (1024, 900, 33, 2), (1025, 255, 602, 0), (2048, 3, 12, 0), (2049, 700, 12, 1), (2047, 1_000_000, 24, 0),
                                              (4096, 256, 40, 0), (5000, 70_000, 128, 0), (20_011, 3, 20, 0), (70_000, 65_537, 16, 0), (40_000, 20_000_000, 4, 0),
                                              (50, 30, 5000, 0), (9, 4, 65_535, 1)])
def test_gradient_sums_by_id(ctx, dtype, n, rows, dim, extra):  # noqa: F811
    rng = np.random.default_rng(n + rows + dim)
    ids = some_ids(rng, n, rows)
    flat, dy = padded(rng.normal(size=(n, dim)), dtype, extra)
    scale = 1.7
    there = (ids >= 0) & (ids < rows)
    names = np.unique(ids[there])
    place = np.full(n, -1)
    place[there] = np.searchsorted(names, ids[there])
    want, size, count = vec.embedding_grad(f64(dy), place, max(len(names), 1), float(np.float32(scale)))
    allowed = ref.sum_error(count[:, None], size) + 2.0 ** -23 * np.abs(want)
    most = min(n, rows)
    few = torch.full((most, dim + extra), PAD, device=DEV)
    touched, met = torch.full((most,), -5, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    ctx.embedding_grad_rows(dy, on_gpu(ids), n, dim, rows, few, touched, met, scale=scale)
    assert int(met) == len(names) and np.array_equal(touched.cpu().numpy()[:len(names)], names) and bool((touched[len(names):] == -5).all())
    check(few[:len(names), :dim], want[:len(names)], allowed[:len(names)], "rows met")
    assert bool((few[len(names):] == PAD).all()) and bool((few[:, dim:] == PAD).all())
    if rows > 1_000_000:
        return
    for out in sorted({F32, dtype}, key=str):
        flat, grad = padded(torch.zeros(rows, dim), out, extra)
        grad.fill_(PAD)
        ctx.embedding_grad(dy, on_gpu(ids), n, dim, rows, grad, scale=scale)
        got = f64(grad)
        check(got[names], want[:len(names)], allowed[:len(names)] + ref.stored(want[:len(names)], out), "named rows")
        got[names] = 0.0
        assert (got == 0.0).all() and untouched(flat, grad)
        before = torch.from_numpy(rng.normal(size=(rows, dim))).to(out)
        grad.copy_(before)
        ctx.embedding_grad(dy, on_gpu(ids), n, dim, rows, grad, scale=scale, add=True)
        sums = want[:len(names)] + f64(before)[names]
        check(f64(grad)[names], sums, allowed[:len(names)] + 2.0 ** -23 * np.abs(f64(before)[names]) + ref.stored(sums, out), "named rows, added to")
        rest = np.setdiff1d(np.arange(rows), names)
        assert np.array_equal(f64(grad)[rest], f64(before)[rest]) and untouched(flat, grad)


def test_rows_of_padding_add_nothing_whatever_they_hold(ctx):  # noqa: F811
    n, dim, rows = 600, 24, 5
    ids = np.arange(n) % (rows + 2) - 1
    dy = torch.ones(n, dim, device=DEV)
    dy[torch.from_numpy((ids < 0) | (ids >= rows)).to(DEV)] = float("nan")
    grad = torch.full((rows, dim), PAD, device=DEV)
    ctx.embedding_grad(dy, on_gpu(ids), n, dim, rows, grad)
    assert np.array_equal(f64(grad), np.bincount(ids[(ids >= 0) & (ids < rows)], minlength=rows)[:, None] * np.ones(dim))


def test_no_id_in_the_table(ctx):  # noqa: F811
    dy, ids = torch.full((700, 8), float("nan"), device=DEV), on_gpu(np.full(700, -1))
    grad = torch.full((9, 8), PAD, device=DEV)
    ctx.embedding_grad(dy, ids, 700, 8, 9, grad, add=True)
    assert bool((grad == PAD).all())
    touched, met = torch.full((9,), -5, dtype=torch.int32, device=DEV), torch.full((1,), 77, dtype=torch.int32, device=DEV)
    ctx.embedding_grad_rows(dy, ids, 700, 8, 9, grad, touched, met)
    assert int(met) == 0 and bool((grad == PAD).all()) and bool((touched == -5).all())
    ctx.embedding_grad(dy, ids, 700, 8, 9, grad)
    assert bool((grad == 0).all())
    met.fill_(77)
    ctx.embedding_grad_rows(dy, ids, 0, 8, 9, grad, touched, met)
    assert int(met) == 0


@pytest.mark.parametrize("n,rows", [(300_001, 1), (200_003, 47), (150_000, 1_000_000)])
def test_long_runs_are_exact_on_whole_numbers_and_the_same_each_time(ctx, n, rows):  # noqa: F811
    """Sums of small whole numbers are exact in whatever order; of others they have one order."""
    rng = np.random.default_rng(n)
    ids, dim = some_ids(rng, n, rows, pad=0.02), 20
    whole = rng.integers(-8, 9, size=(n, dim)).astype(np.float64)
    want, _, _ = vec.embedding_grad(whole, ids, rows, 1.0)
    grad = torch.full((rows, dim), PAD, device=DEV)
    ctx.embedding_grad(torch.from_numpy(whole).to(torch.bfloat16).to(DEV), on_gpu(ids), n, dim, rows, grad)
    assert np.array_equal(f64(grad), want)
    dy, at = torch.from_numpy(rng.normal(size=(n, dim))).float().to(DEV), on_gpu(ids)
    again = torch.empty_like(grad)
    ctx.embedding_grad(dy, at, n, dim, rows, grad, scale=0.3)
    ctx.embedding_grad(dy, at, n, dim, rows, again, scale=0.3)
    assert torch.equal(grad, again)


def test_far_rows_of_a_large_table(ctx):  # noqa: F811
    """Offsets beyond 32 bits."""
    rows, dim = 9_000_001, 256                             # 2.3 G numbers of 2 bytes
    table = torch.zeros(rows, dim, dtype=torch.bfloat16, device=DEV)
    ids = np.array([rows - 1, 0, 8_388_607, 8_388_608, rows - 1, 8_500_000])
    table[torch.from_numpy(ids).to(DEV)] = torch.arange(6, dtype=torch.bfloat16, device=DEV)[:, None] + 1.0
    want = table[torch.from_numpy(ids).to(DEV)].clone()
    y = torch.empty(6, dim, dtype=torch.bfloat16, device=DEV)
    ctx.embedding(table, rows, on_gpu(ids), 6, dim, y)
    assert torch.equal(y, want)
    ctx.embedding_grad(y, on_gpu(ids), 6, dim, rows, table)
    got = table[torch.from_numpy(ids).to(DEV)].float()
    assert torch.equal(got[1], want[1].float()) and torch.equal(got[0], 2.0 * want[0].float()) and float(table[5].float().abs().max()) == 0.0
    assert torch.equal(got[5], want[5].float()) and torch.equal(got[3], want[3].float())


def test_gradients_recorded_into_a_graph(ctx):  # noqa: F811
    rng = np.random.default_rng(3)
    n, rows, dim = 3000, 500, 36
    side = torch.cuda.Stream()
    dy, grad, few = torch.zeros(n, dim, device=DEV), torch.zeros(rows, dim, device=DEV), torch.zeros(rows, dim, device=DEV)
    ids, y = torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros(n, dim, device=DEV)
    touched, met = torch.zeros(rows, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)

    def calls(grad, few, touched, met, y, stream):
        ctx.embedding_grad(dy, ids, n, dim, rows, grad, scale=0.5, stream=stream)
        ctx.embedding_grad_rows(dy, ids, n, dim, rows, few, touched, met, scale=0.5, stream=stream)
        ctx.embedding(grad, rows, ids, n, dim, y, stream=stream)
    with torch.cuda.stream(side):
        calls(grad, few, touched, met, y, side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls(grad, few, touched, met, y, torch.cuda.current_stream())
    for turn in range(3):
        dy.copy_(torch.from_numpy(rng.normal(size=(n, dim))))
        ids.copy_(on_gpu(some_ids(rng, n, rows)))
        graph.replay()
        torch.cuda.synchronize()
        eager = [torch.zeros_like(t) for t in (grad, few, touched, met, y)]
        if turn == 0:
            few.zero_(), touched.zero_()
            graph.replay()
        calls(*eager, None)
        torch.cuda.synchronize()
        k = int(met)
        assert torch.equal(grad, eager[0]) and torch.equal(few[:k], eager[1][:k]) and torch.equal(touched[:k], eager[2][:k])
        assert torch.equal(met, eager[3]) and torch.equal(y, eager[4])


def test_lookup_gradient_against_differences(ctx):  # noqa: F811
    """d/dt of sum(dy . lookup(table + t direction)) is sum(grad . direction): the lookup is linear, so one step says it."""
    rng = np.random.default_rng(8)
    n, rows, dim = 400, 60, 50
    ids = on_gpu(some_ids(rng, n, rows))
    table, direction = (torch.from_numpy(rng.integers(-8, 9, size=(rows, dim))).float().to(DEV) for _ in range(2))
    dy = torch.from_numpy(rng.integers(-4, 5, size=(n, dim))).float().to(DEV)
    y0, y1, grad = torch.empty(n, dim, device=DEV), torch.empty(n, dim, device=DEV), torch.empty(rows, dim, device=DEV)
    ctx.embedding(table, rows, ids, n, dim, y0, scale=4.0)
    ctx.embedding(table + direction, rows, ids, n, dim, y1, scale=4.0)
    ctx.embedding_grad(dy, ids, n, dim, rows, grad, scale=4.0)
    assert float((dy.double() * (y1 - y0).double()).sum()) == float((grad.double() * direction.double()).sum())


@pytest.mark.parametrize("n,rows", [(5000, 7), (5000, 3000), (100_003, 7), (100_003, 70_000)])
def test_gradients_of_many_entries_count_on_the_device(ctx, n, rows):  # noqa: F811
    """Whole numbers, whose sums are exact in any order; ids and rows behind the count hold what would show."""
    dim = 12
    rng = np.random.default_rng(n + rows)
    ids, dy = some_ids(rng, n, rows), rng.integers(-8, 9, size=(n, dim)).astype(np.float64)
    for live in (0, 1, 2049, n - 1, n, n + 5):
        count = min(live, n)
        want = np.zeros((rows, dim))
        there = (ids[:count] >= 0) & (ids[:count] < rows)
        np.add.at(want, ids[:count][there], dy[:count][there])
        t = torch.from_numpy(dy).float().to(DEV)
        t[count:] = float("nan")
        n_dev = torch.tensor([live], dtype=torch.int32, device=DEV)
        table = torch.full((rows + 1, dim + 3), PAD, device=DEV)
        ctx.embedding_grad(t, on_gpu(ids), n, dim, rows, table[:rows, :dim], n_dev=n_dev)
        assert np.array_equal(f64(table[:rows, :dim]), want) and bool((table[rows] == PAD).all()) and bool((table[:, dim:] == PAD).all())
        most = min(n, rows)
        grad, touched, met = torch.full((most, dim), PAD, device=DEV), torch.full((most,), -7, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        ctx.embedding_grad_rows(t, on_gpu(ids), n, dim, rows, grad, touched, met, n_dev=n_dev)
        named = np.unique(ids[:count][there])
        assert int(met) == len(named) and np.array_equal(touched.cpu().numpy()[:len(named)], named) and bool((touched[len(named):] == -7).all())
        assert np.array_equal(f64(grad)[:len(named)], want[named]) and bool((grad[len(named):] == PAD).all())
