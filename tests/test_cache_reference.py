"""The float64 definitions of the operators around the cache, checked against what they have to satisfy (CPU)."""
import numpy as np
import pytest

import cache_reference as ref


def inputs(seed, T=5, H=3, D=64, rot=32):
    g = np.random.default_rng(seed)
    return g.standard_normal((T, H, D)), 1 + 0.3 * g.standard_normal(D), g.integers(-50, 5000, T), 1e4 ** (-np.arange(0, rot, 2) / max(rot, 1))


@pytest.mark.parametrize("interleaved", [False, True])
def test_scores_depend_on_distance_alone(interleaved):
    x, w, pos, f = inputs(1)
    y = x[:, ::-1]
    a = np.einsum("thd,thd->th", ref.rotate(x, pos, f, interleaved), ref.rotate(y, pos + 7, f, interleaved))
    b = np.einsum("thd,thd->th", ref.rotate(x, pos + 900, f, interleaved), ref.rotate(y, pos + 907, f, interleaved))
    np.testing.assert_allclose(a, b, rtol=1e-9, atol=1e-9)
    np.testing.assert_allclose(ref.rotate(ref.rotate(x, pos, f, interleaved), pos, f, interleaved, back=True), x, atol=1e-12)


def test_unit_rms():
    x, w, pos, f = inputs(2)
    y, r = ref.norm(x, np.ones(64), 0.0)
    np.testing.assert_allclose((y * y).mean(-1), 1.0)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("normed", [False, True])
def test_gradient_against_differences(interleaved, normed):
    x, w, pos, f = inputs(3, T=2, H=2)
    w = w if normed else None
    dz = np.random.default_rng(4).standard_normal(x.shape)
    loss = lambda x, w: (ref.qk_rope(x, w, 1e-3, pos, f, interleaved)[0] * dz).sum()
    dx, _, dw, _ = ref.qk_rope_backward(x, w, 1e-3, pos, f, interleaved, dz)
    h = 1e-6
    for at in [(0, 0, 0), (1, 1, 63), (0, 1, 17), (1, 0, 40)]:
        e = np.zeros_like(x)
        e[at] = h
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * h) - dx[at]) < 1e-7
    if normed:
        for i in (0, 33, 63):
            e = np.zeros_like(w)
            e[i] = h
            assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * h) - dw[i]) < 1e-7


def test_bf16_rounding():
    x = np.array([1.0, 1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, -3.14159, 0.0])
    np.testing.assert_array_equal(ref.bf16(x), [1.0, 1.0, 1 + 2.0 ** -6, -3.140625, 0.0])


def test_eviction_keeps_the_heaviest_in_order():
    w = np.array([0.0, 5.0, 1.0, 5.0, 0.0, 2.0, 0.5, 9.0])
    assert ref.evict(w, 8, 8, 0, 0) == list(range(8))
    assert ref.evict(w, 8, 3, 0, 0) == [1, 3, 7]
    assert ref.evict(w, 8, 3, 1, 1) == [0, 1, 7]
    assert ref.evict(w, 6, 4, 0, 2) == [1, 3, 4, 5]
    assert ref.evict(w, 8, 2, 0, 2) == [6, 7]
    assert ref.evict(np.array([1.0, np.nan, 3.0, -0.0, 0.0]), 5, 3, 0, 0) == [0, 1, 2]
    assert ref.evict(np.array([-0.0, 0.0, -1.0, 0.0]), 4, 2, 0, 0) == [0, 1]
