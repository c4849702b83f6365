"""The plain implementations of the layers in front of a loss, held to differences and to what is published."""
import numpy as np
import pytest

from tests import layers_reference as ref


def _difference(f, x, step=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += step
        b[i] -= step
        g[i] = (f(a) - f(b)) / (2 * step)
    return g


@pytest.mark.parametrize("kind", [ref.NONE, ref.RELU, ref.GELU, ref.SILU])
def test_linear_gradients_are_the_differences(kind):
    rng = np.random.default_rng(kind)
    x, w, b, dy = rng.normal(size=(3, 4)), rng.normal(size=(5, 4)), rng.normal(size=5), rng.normal(size=(3, 5))
    z = ref.linear(x, w, b)[1]
    dx, dw, db = ref.linear_grad(dy, x, w, z, kind)
    assert np.allclose(dx, _difference(lambda v: (dy * ref.linear(v, w, b, kind=kind)[0]).sum(), x), atol=1e-7)
    assert np.allclose(dw, _difference(lambda v: (dy * ref.linear(x, v, b, kind=kind)[0]).sum(), w), atol=1e-7)
    assert np.allclose(db, _difference(lambda v: (dy * ref.linear(x, w, v, kind=kind)[0]).sum(), b), atol=1e-7)


def test_cross_entropy_gradients_are_the_differences():
    rng = np.random.default_rng(9)
    x, w = rng.normal(size=(4, 3)), rng.normal(size=(6, 3))
    target, weight = np.array([2, -1, 5, 0]), np.array([0.5, 1.0, 2.0, 0.0])
    loss, lse, dx, dw, _ = ref.xent(x, w, target, weight)
    assert loss[1] == loss[3] == lse[1] == 0 and not dx[1].any() and not dx[3].any()
    assert np.allclose(dx, _difference(lambda v: ref.xent(v, w, target, weight)[0].sum(), x), atol=1e-7)
    assert np.allclose(dw, _difference(lambda v: ref.xent(x, v, target, weight)[0].sum(), w), atol=1e-7)


def test_activation_limits():
    z = np.array([-np.inf, -1e30, -0.0, 0.0, 1e30, np.inf])
    for kind in (ref.GELU, ref.SILU):
        with np.errstate(over="ignore"):
            assert ref.act(z, kind).tolist() == [0, 0, 0, 0, 1e30, np.inf]
            assert np.allclose(ref.slope(z, kind)[[0, 1, 4, 5]], [0, 0, 1, 1])


def test_philox_gives_the_published_numbers():
    """The known answers that come with the paper's generator: counter and key of zeros, of ones, and of digits of pi."""
    assert ref.philox(0, 0, 0) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = (1 << 64) - 1
    assert ref.philox(ones, ones, ones) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert ref.philox(0x85A308D3243F6A88, 0x0370734413198A2E, 0x299F31D0A4093822) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_kept_share():
    keep, scale = ref.kept(80000, 0.25, 7, 3)
    assert scale == 4 / 3 and abs(keep.mean() - 0.75) < 6 * (0.25 * 0.75 / 80000) ** 0.5
    assert ref.kept(16, 0.0, 1, 1)[0].all() and not ref.kept(16, 1.0, 1, 1)[0].any()
