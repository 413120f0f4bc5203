"""The 64-bit forms of the training step's operators: pins by hand, gradients against differences."""
import numpy as np
import pytest

import training_reference as ref


def test_codes_by_hand():
    x = np.zeros((1, 40))
    x[0, :10] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.1, -6.0, -0.1]         # largest 6: scale 1; halves go to the even code
    x[0, 32:36] = [7.9, -7.0, 3.0, -0.0]                                        # largest 7.9: scale 1, above 6 to 6
    packed, values = ref.quantize(x)
    assert packed.shape == (1, 36) and ref.words(40) == 9
    assert packed[0, :5].tolist() == [0x20, 0x42, 0x64, 0x76, 0x8F]
    assert values[0, :10].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, -6.0, 0.0]
    assert values[0, 32:36].tolist() == [6.0, -6.0, 3.0, 0.0] and packed[0, 17] == 0x85
    assert packed[0, 32:36].tolist() == [127, 127, 0, 0]
    assert np.array_equal(ref.dequantize(packed, 40), values)


def test_scales_of_the_largest_the_smallest_and_what_is_not_finite():
    x = np.zeros((6, 32))
    x[0, 3] = 3.4e38
    x[1, 3] = 2.0 ** -149
    x[2, 3] = np.inf
    x[3, 3] = np.nan
    x[4, 3] = 2.0 ** -126
    packed, values = ref.quantize(x)
    assert packed[:, 16].tolist() == [252, 0, 255, 255, 0, 0]
    assert values[0, 3] == 6 * 2.0 ** 125 and values[1, 3] == 0 and np.isnan(values[2:4]).all()
    assert values[4, 3] == 2.0 ** -126 and not values[5].any()
    assert np.array_equal(ref.dequantize(packed, 32), values, equal_nan=True)


@pytest.mark.parametrize("gamma", [True, False])
def test_layer_norm_gradient_is_the_difference_quotient(gamma):
    rng = np.random.default_rng(3)
    n, dim, eps, step = 3, 7, 1e-5, 1e-6
    x, dy = rng.normal(size=(n, dim)), rng.normal(size=(n, dim))
    g, b = (rng.normal(size=dim) if gamma else np.ones(dim)), rng.normal(size=dim)
    loss = lambda x, g, b: float((ref.layer_norm(x, g, b, eps)[0] * dy).sum())       # noqa: E731
    _, mean, rstd = ref.layer_norm(x, g, b, eps)
    dx, dg, db = ref.layer_norm_grad(dy, x, g, mean, rstd)
    for i in range(n):
        for k in range(dim):
            d = np.zeros_like(x)
            d[i, k] = step
            assert abs((loss(x + d, g, b) - loss(x - d, g, b)) / (2 * step) - dx[i, k]) < 1e-7
    for k in range(dim):
        d = np.zeros(dim)
        d[k] = step
        assert abs((loss(x, g + d, b) - loss(x, g - d, b)) / (2 * step) - dg[k]) < 1e-7
        assert abs((loss(x, g, b + d) - loss(x, g, b - d)) / (2 * step) - db[k]) < 1e-7


def test_clip_by_hand():
    norm, out = ref.clip([np.array([3.0]), np.array([0.0, -4.0])], 1.0)
    assert norm == 5.0 and np.allclose(out[0], 0.6) and np.allclose(out[1], [0.0, -0.8])
    assert ref.clip([np.array([3.0])], 3.0)[1][0][0] == 3.0
    assert np.isinf(ref.clip([np.array([np.inf, 2.0])], 1.0)[1][0][0])
