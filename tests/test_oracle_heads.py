"""The float64 reference of head norms and rotations: what a rotation is, pair by pair, and gradients
against differences."""
import numpy as np
import pytest

from oracle import heads as oh


@pytest.mark.parametrize("dims,layout", [((8,), "interleaved"), ((8,), "halves"), ((4, 6, 2), "interleaved"),
                                         ((4, 6, 2), "halves"), ((4, 6, 2), "split"), ((2,), "split")])
def test_pairs_cover_the_turned_values_once(dims, layout):
    got = oh.pairs(dims, layout)
    assert sorted(i for p in got for i in p[:2]) == list(range(sum(dims)))
    assert [p[2] for p in got] == [a for a, n in enumerate(dims) for _ in range(n // 2)]


def test_a_rotation_is_a_complex_product_and_depends_on_differences():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 1, 1, 1, 8))
    freqs = 0.3 ** np.arange(4)
    at = lambda p: np.full((1, 1, 1), p)  # noqa: E731
    for layout in ("interleaved", "halves", "split"):
        i, j = np.array(oh.pairs((8,), layout))[:, :2].T
        y = oh.turn(q, at(5), freqs, (8,), layout)
        z = (q[..., i] + 1j * q[..., j]) * np.exp(1j * 5 * freqs)
        assert np.allclose(y[..., i], z.real) and np.allclose(y[..., j], z.imag)
        dots = [(oh.turn(q, at(5 + s), freqs, (8,), layout) * oh.turn(k, at(2 + s), freqs, (8,), layout)).sum()
                for s in (0, 7, 1000)]
        assert np.allclose(dots, dots[0])
        assert np.allclose(oh.turn(y, at(5), freqs, (8,), layout, back=True), q)


def test_norms_by_hand():
    x = np.array([[[[3.0, 4.0]]]])
    y, r = oh.normed(x, "rms", 0.0)
    assert np.allclose(y, x / np.sqrt(12.5)) and np.allclose(r, 1 / np.sqrt(12.5))
    assert np.allclose(oh.normed(x, "layer", 0.0)[0], [[[[-1.0, 1.0]]]])
    assert np.array_equal(oh.normed(x, None, 0.0)[0], x)


@pytest.mark.parametrize("norm", [None, "rms", "layer"])
@pytest.mark.parametrize("layout", [None, "interleaved", "halves", "split"])
def test_gradients_against_differences(norm, layout):
    rng = np.random.default_rng(3)
    x, dy = rng.standard_normal((2, 3, 2, 8)), rng.standard_normal((2, 2, 3, 8))
    how = dict(norm=norm, eps=1e-3, lens=[3, 2])
    if norm:
        how["weight"] = 1 + 0.3 * rng.standard_normal(8)
    if norm == "layer":
        how["bias"] = rng.standard_normal(8)
    if layout:
        how.update(positions=rng.integers(0, 9, (2, 3, 2)), freqs=rng.random(3), dims=(4, 2), layout=layout)
    dx, dw, db = oh.backward(x, dy, **how)

    def slope(name, base, step):
        hi, lo = ((oh.forward(**{**dict(x=x), **how, name: base + s * step}) * dy).sum() for s in (1e-5, -1e-5))
        return (hi - lo) / 2e-5

    step = rng.standard_normal(x.shape)
    assert np.isclose(slope("x", x, step), (dx * step).sum(), rtol=1e-6, atol=1e-8)
    assert not dx[1, 2].any()
    step = rng.standard_normal(8)
    if norm:
        assert np.isclose(slope("weight", how["weight"], step), (dw * step).sum(), rtol=1e-6)
    if norm == "layer":
        assert np.isclose(slope("bias", how["bias"], step), (db * step).sum(), rtol=1e-6)
