"""The plain implementations that the operators are tested against, held against hand-worked values and differences."""
import numpy as np
import pytest

from tests import operators_reference as ref


def test_rounding_of_every_magnitude_and_tie_by_hand():
    # the largest element 6 sets the scale to 2^(2 - 2) = 1
    v = np.zeros(32)
    v[:16] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 5.5, -0.25, -0.75, 0.2500001, 1.2499, -2.4999, 4.9, -6]
    codes, byte = ref.mx4_block(v)
    assert byte == 127
    want = [6, 0, 1, 1, 2, 2, 4, 4, 6, 0, -1, 0.5, 1, -2, 4, -6]
    assert ref.mx4_values(codes[None, :].repeat(4, 0).reshape(1, 128), np.full((1, 4), byte))[0, :16].tolist() == want


def test_values_beyond_six_saturate_and_scales_follow_the_exponent():
    v = np.zeros(32)
    v[0], v[1] = 7.99, 1.0
    codes, byte = ref.mx4_block(v)
    assert byte == 127 and codes[0] == 7 and codes[1] == 2
    v[0] = 8.0
    codes, byte = ref.mx4_block(v)
    assert byte == 128 and codes[0] == 6 and codes[1] == 1
    assert ref.mx4_block(np.zeros(32))[1] == 0
    v[0] = 2.0 ** -140                                       # the smallest scale is 2^-127
    assert ref.mx4_block(v * 0 + 2.0 ** -140)[1] == 0
    v[0] = np.inf
    assert ref.mx4_block(v)[1] == 255


def test_pack_and_unpack_are_inverse():
    rng = np.random.default_rng(0)
    codes, byte = rng.integers(0, 16, (5, 384)), rng.integers(0, 253, (5, 12))
    c, b = ref.mx4_unpack(*ref.mx4_pack(codes, byte))
    assert np.array_equal(c, codes) and np.array_equal(b, byte)


@pytest.mark.parametrize("T", [0.5, 1.0, 3.0])
def test_distillation_gradient_against_differences(T):
    rng = np.random.default_rng(1)
    z, t = rng.normal(0, 2, (3, 9)), rng.normal(0, 2, (3, 4))
    idx = np.array([[1, 5, 8, 2], [0, 3, 3, 9], [4, -1, -1, -1]])      # twice the same, outside, padding
    w = np.array([1.0, 0.5, 2.0])
    _, _, grad = ref.distill(z, idx, t, T, w)
    step = 1e-6
    for r in range(3):
        for v in range(9):
            up, down = z.copy(), z.copy()
            up[r, v] += step
            down[r, v] -= step
            d = (ref.distill(up, idx, t, T, w)[0].sum() - ref.distill(down, idx, t, T, w)[0].sum()) / (2 * step)
            assert abs(d - grad[r, v]) < 1e-7 * max(1.0, T * T)
    assert np.allclose(grad.sum(1), 0)
