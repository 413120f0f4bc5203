"""The long loops of the training step's sums over rows, on numbers whose sums are exact in 32 bits whatever their order: every row counts, so that
results are compared bit by bit.

Sizes are written for 256 compute units, where the ranges of rows that the weight gradient deals out are as long as the comments say; on another device the
ranges differ and the results do not."""
import numpy as np
import pytest
import torch

import training_reference as ref
from test_gpu_training_ops import DEV, F32, PAD, _name_the_case, ctx     # noqa: F401  (fixtures among them)

pytestmark = pytest.mark.gpu

# rows, numbers of a row, outputs, rows counted on the device (None: all)
GRADIENTS = [
    # 256 columns to a tile, 64 rows to a step: ranges of two, three, four and seven steps; the last one shorter, with a rest and without
    (16_384, 256, 256, None), (24_576, 256, 256, None), (24_525, 256, 256, None), (32_768, 256, 256, None), (32_767, 256, 256, None),
    (57_344, 256, 256, None), (57_343, 256, 256, None), (57_217, 256, 256, None), (57_280, 256, 256, 50_001), (24_576, 256, 256, 64),
    (5376, 602, 130, None), (8034, 602, 130, None), (18_753, 602, 130, None), (18_816, 602, 130, 9001),
    # 128 columns
    (32_768, 100, 128, None), (49_100, 100, 128, None), (65_535, 128, 258, None), (100_003, 64, 70, None), (38_016, 33, 200, 30_030),
    # up to 64 outputs, 32 rows to a step of a wavefront: one, three, five and sixteen steps
    (20_000, 100, 41, None), (150_001, 100, 41, None), (150_001, 100, 3, None), (40_003, 602, 47, None), (100_003, 602, 41, None), (60_000, 256, 64, 41_234),
    (131_072, 100, 64, None), (30_000, 17, 7, None),
    # so many tiles that each has one range: two, three and seven steps, then of wavefronts of up to 64 outputs
    (128, 4200, 1030, None), (197, 4200, 1030, None), (511, 4200, 1030, None), (800, 17_000, 41, None),
]


def packed_codes(n, dim, seed):
    """(packed rows with every scale 1, their numbers float32): every code there is."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    groups = -(-dim // 32)
    code = torch.randint(0, 16, (n, groups * 32), generator=gen, device=DEV, dtype=torch.uint8)
    code[:, dim:] = 0
    return pack(code, groups), code_values(code)[:, :dim]


def pack(code, groups):
    n = code.shape[0]
    out = torch.zeros(n, 4 * ref.words(groups * 32), dtype=torch.uint8, device=DEV)
    out[:, :16 * groups] = code[:, 0::2] + 16 * code[:, 1::2]
    out[:, 16 * groups:17 * groups] = 127
    return out.view(F32)


def code_values(code):
    table = torch.from_numpy(np.concatenate([ref.MAGNITUDES, -ref.MAGNITUDES])).float().to(DEV)
    return table[code.int()]


def whole_numbers(shape, dtype, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(-8, 9, shape, generator=gen, device=DEV).to(dtype)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,dim,out,live", GRADIENTS)
def test_gradient_counts_every_row_of_every_step(ctx, dtype, n, dim, out, live):
    """dy of whole numbers up to 8, rows of multiples of 0.5 up to 6: sums of up to 150,001 of their products are multiples of 0.5 below 2^23, and exact."""
    real = n if live is None else live
    rows, values = packed_codes(n, dim, n + dim)
    dy = whole_numbers((n, out), dtype, out)
    n_dev = None if live is None else torch.tensor([live], dtype=torch.int32, device=DEV)
    grad = torch.full((out, dim), PAD, device=DEV)
    ctx.mx4_matmul_grad(dy, rows, n, out, dim, grad, n_dev=n_dev)
    want = dy[:real].double().t().contiguous() @ values[:real].double()
    assert float(want.abs().max()) < 2.0 ** 23
    assert torch.equal(grad.double(), want)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,dim,out,live", GRADIENTS + [(1, 32, 70, None), (1, 256, 70, None), (63, 256, 130, None)])
def test_gradient_keeps_all_bits_of_dy_in_every_step(ctx, dtype, n, dim, out, live):
    """One row of each column is 1 or -1, the others are 0: the gradient is that row's dy, in all its bits."""
    real = n if live is None else live
    gen = torch.Generator(device=DEV).manual_seed(n + dim + out)
    column = torch.arange(dim, device=DEV)
    chosen = (column * (real // dim + 1) + torch.randint(0, real, (dim,), generator=gen, device=DEV) % (real // dim + 1)) % real
    groups = -(-dim // 32)
    code = torch.zeros(n, groups * 32, dtype=torch.uint8, device=DEV)
    code[chosen, column] = (2 + 8 * (column % 2)).to(torch.uint8)
    # every bit of the number set at random; 32-bit numbers of 2^-40 to 2^40, 16-bit ones of every exponent but the last
    if dtype == F32:
        mantissa = torch.randint(0, 1 << 24, (n, out), generator=gen, device=DEV)
        power = torch.randint(87, 168, (n, out), generator=gen, device=DEV)
        dy = ((mantissa & 0x7FFFFF) | (power << 23) | ((mantissa >> 23) << 31)).to(torch.int64)
        dy = torch.where(dy >= 1 << 31, dy - (1 << 32), dy).to(torch.int32).view(F32)
    else:
        dy = torch.randint(-(1 << 15), 1 << 15, (n, out), generator=gen, device=DEV).to(torch.int16).view(dtype)
        dy = torch.where(torch.isfinite(dy), dy, torch.ones_like(dy))
    n_dev = None if live is None else torch.tensor([live], dtype=torch.int32, device=DEV)
    grad = torch.full((out, dim), PAD, device=DEV)
    ctx.mx4_matmul_grad(dy, pack(code, groups), n, out, dim, grad, n_dev=n_dev)
    want = dy[chosen].float().t() * torch.where(column % 2 == 0, 1.0, -1.0)
    assert torch.equal(grad, want)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("n,dim", [(70_001, 64), (200_003, 100), (60_001, 256), (100_003, 602), (30_011, 1000), (40_009, 1024), (20_011, 1025), (9007, 2049), (40_001, 3),
                                   (250_000, 16), (513, 255), (100_000, 33)])
def test_layer_norm_gradient_counts_every_row(ctx, dtype, n, dim):
    """With mean 0 and deviation 1 h is x: the gain's gradient is a sum of whole numbers up to 64, the bias's of up to 8."""
    x, dy = whole_numbers((n, dim), dtype, n), whole_numbers((n, dim), dtype, dim)
    dg, db = torch.full((dim,), PAD, device=DEV), torch.full((dim,), PAD, device=DEV)
    dx = torch.empty(n, dim, dtype=dtype, device=DEV)
    for room, live in ((n, None), (n, n - n // 3)):
        real = room if live is None else live
        n_dev = None if live is None else torch.tensor([live], dtype=torch.int32, device=DEV)
        ctx.layer_norm_grad(dy, x, room, dim, None, torch.zeros(n, device=DEV), torch.ones(n, device=DEV), dx, dg, db, n_dev=n_dev)
        assert torch.equal(dg.double(), (dy[:real].double() * x[:real].double()).sum(0))
        assert torch.equal(db.double(), dy[:real].double().sum(0))
