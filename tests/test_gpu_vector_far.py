"""Lookup of learned vectors and its gradient on an MI355X at the lengths where the kernels go around their loops again: more than 1048576 entries (a digit's counts
are added up in a second round), more than 4194304 (a workgroup sorts a second tile), and results beyond 32 MiB, which are stored past the caches."""
import pytest
import torch

import training_reference as ref
from test_gpu_training_ops import DEV, F32, PAD, ctx, untouched, _name_the_case  # noqa: F401  (fixtures among them)

pytestmark = pytest.mark.gpu


def entries(n, rows, dim, dtype, seed):
    """(ids, dy, which ids are in the table): hubs often, some ids not in the table; whole numbers up to 8 of both signs, whose sums stay below 2^24 and are exact in any order."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    u = torch.rand((n,), generator=gen, device=DEV, dtype=torch.float64)
    ids = (u.pow(3) * rows).long().clamp(max=rows - 1)
    gone = torch.rand((n,), generator=gen, device=DEV) < 0.03
    strange = torch.tensor([-1, rows, 2 ** 31 - 1, -2 ** 31], device=DEV)[torch.randint(0, 4, (n,), generator=gen, device=DEV)]
    ids = torch.where(gone, strange, ids)
    dy = torch.randint(-8, 9, (n, dim), generator=gen, device=DEV).to(dtype)
    there = (ids >= 0) & (ids < rows)
    return ids.int(), dy, there


def sums(ids, dy, there, rows):
    """Whole numbers: differences of a running sum over the entries in the order of their ids."""
    at, order = torch.sort(ids[there].long())
    running = torch.cat([torch.zeros((1, dy.shape[1]), dtype=torch.int64, device=DEV), dy[there][order].long().cumsum(0)])
    ends = torch.searchsorted(at, torch.arange(rows, device=DEV), right=True)
    until = running[ends]
    return (until - torch.cat([torch.zeros_like(until[:1]), until[:-1]])).double()


@pytest.mark.parametrize("n", [1_048_577 + 333, 4_194_304, 4_194_305 + 70_001])
@pytest.mark.parametrize("rows,dim,dtype", [(1000, 4, F32), (3_000_000, 5, torch.bfloat16), (200, 9, torch.float16)])
def test_gradients_of_more_entries_than_one_round_takes(ctx, n, rows, dim, dtype):  # noqa: F811
    ids, dy, there = entries(n, rows, dim, dtype, n + rows)
    for live in (n, n - 12_345):
        n_dev = None if live == n else torch.tensor([live], dtype=torch.int32, device=DEV)
        inside = there & (torch.arange(n, device=DEV) < live)
        want = sums(ids, dy, inside, rows)
        grad = torch.full((rows + 1, dim), PAD, device=DEV)
        ctx.embedding_grad(dy, ids, n, dim, rows, grad[:rows], n_dev=n_dev)
        assert torch.equal(grad[:rows].double(), want) and bool((grad[rows] == PAD).all())
        most = min(n, rows)
        grad = torch.full((most, dim), PAD, device=DEV)
        touched, met = torch.full((most,), -7, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        ctx.embedding_grad_rows(dy, ids, n, dim, rows, grad, touched, met, n_dev=n_dev)
        named = torch.unique(ids[inside])
        k = named.numel()
        assert int(met) == k and torch.equal(touched[:k], named) and bool((touched[k:] == -7).all())
        assert torch.equal(grad[:k].double(), want[named.long()]) and bool((grad[k:] == PAD).all())


@pytest.mark.parametrize("table_type", ref.TYPES)
@pytest.mark.parametrize("out", ref.TYPES)
@pytest.mark.parametrize("n,dim,extra", [(300_001, 64, 0), (140_003, 128, 8), (1_050_000, 16, 0), (66_000, 264, 0)])
def test_lookups_whose_result_is_stored_past_the_caches(ctx, table_type, out, n, dim, extra):  # noqa: F811
    """Times 4, which is exact: the same numbers as torch's indexing, rounded once."""
    rows = 50_000
    gen = torch.Generator(device=DEV)
    gen.manual_seed(n)
    table = torch.randn(rows, dim, generator=gen, device=DEV).to(table_type)
    ids = torch.randint(-2000, rows + 2000, (n,), generator=gen, device=DEV)
    flat = torch.full(((n + 1) * (dim + extra),), PAD, dtype=out, device=DEV)
    y = torch.as_strided(flat, (n, dim), (dim + extra, 1))
    assert y.data_ptr() % 16 == 0 and (dim + extra) * y.element_size() % 16 == 0 and n * dim * y.element_size() > 32 << 20
    ctx.embedding(table, rows, ids.int(), n, dim, y, scale=4.0)
    there = (ids >= 0) & (ids < rows)
    want = torch.where(there[:, None], table[ids.clamp(0, rows - 1)].float() * 4.0, torch.zeros((), device=DEV)).to(out)
    assert torch.equal(y, want) and untouched(flat, y)


@pytest.mark.parametrize("n,rows", [(50_001, 1), (50_001, 3), (16_384 * 4 - 1, 4), (16_384 * 4, 4), (400_003, 5), (1_500_000, 47)])
@pytest.mark.parametrize("dim,dtype", [(32, F32), (33, F32), (40, torch.bfloat16), (100, torch.float16), (300, F32), (1030, torch.bfloat16)])
def test_gradients_of_few_ids_that_have_all_entries(ctx, n, rows, dim, dtype):  # noqa: F811
    """Both sides of the line beyond which ids are joined by narrow groups, and hubs of many pieces."""
    if n * dim > 200_000_000:
        n = 200_000_000 // dim
    ids, dy, there = entries(n, rows, dim, dtype, n + dim)
    want = sums(ids, dy, there, rows)
    grad = torch.full((rows + 1, dim), PAD, device=DEV)
    ctx.embedding_grad(dy, ids, n, dim, rows, grad[:rows])
    assert torch.equal(grad[:rows].double(), want) and bool((grad[rows] == PAD).all())
    many = torch.full((rows, dim), PAD, device=DEV)
    touched, met = torch.full((rows,), -7, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    ctx.embedding_grad_rows(dy, ids, n, dim, rows, many, touched, met)
    named = torch.unique(ids[there])
    k = named.numel()
    assert int(met) == k and torch.equal(touched[:k], named) and torch.equal(many[:k].double(), want[named.long()])
