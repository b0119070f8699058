"""Pins of the oracles of routing and of 8-bit products: closed forms, brute force, differences."""
import itertools

import numpy as np
import pytest

from oracle import i8, route


def test_softmax_choice_by_hand():
    z = np.log(np.array([[1.0, 4.0, 2.0, 3.0]]))
    ids, w, _ = route.choose(z, 2, renorm=False)
    assert ids.tolist() == [[1, 3]] and np.allclose(w, [[0.4, 0.3]], rtol=1e-14)
    ids, w, _ = route.choose(z, 2, renorm=True, scale=7.0)
    assert np.allclose(w, [[4.0, 3.0]], rtol=1e-14)


def test_bias_moves_the_choice_and_not_the_weights():
    z = np.array([[0.0, 1.0, -1.0]])
    s = 1 / (1 + np.exp(-z))
    ids, w, _ = route.choose(z, 1, route.SIGMOID, bias=[0.0, 0.0, 1.0], renorm=False)
    assert ids.tolist() == [[2]] and np.allclose(w, s[:, 2:])
    assert route.choose(z, 1, route.SIGMOID, bias=[0.0, np.nan, -np.inf])[0].tolist() == [[0]]


def test_groups_against_all_subsets():
    rng = np.random.default_rng(1)
    z, bias = rng.normal(size=(20, 12)), rng.normal(size=12) * 0.1
    s = 1 / (1 + np.exp(-z))
    ids, _, _ = route.choose(z, 4, route.SIGMOID, bias, groups=4, top_groups=2, group_top=2)
    for t in range(20):
        key = s[t] + bias
        groups = max(itertools.combinations(range(4), 2), key=lambda c: sum(np.sort(key[3 * g:3 * g + 3])[-2:].sum() for g in c))
        allowed = [e for e in range(12) if e // 3 in groups]
        assert sorted(ids[t]) == sorted(sorted(allowed, key=lambda e: -key[e])[:4])


def test_closed_experts_and_ties():
    z = np.array([[-np.inf] * 4, [-np.inf, 2.0, np.nan, 2.0], [np.inf, 1.0, 0.0, np.inf]])
    ids, w, _ = route.choose(z, 3)
    assert ids.tolist() == [[-1, -1, -1], [1, 3, -1], [0, 3, 1]]
    assert np.array_equal(w, [[0, 0, 0], [0.5, 0.5, 0], [0.5, 0.5, 0]])


def test_dispatch_is_a_stable_sort():
    ids = np.array([[1, 0], [1, 2], [-1, -1], [0, 1]])
    counts, offsets, place, source = route.dispatch(ids, 4, 4, 16)
    assert counts.tolist() == [2, 3, 1, 0] and offsets.tolist() == [0, 4, 8, 12, 12]
    assert place.tolist() == [4, 0, 5, 8, -1, -1, 1, 6]
    assert source.tolist() == [1, 6, -1, -1, 0, 2, 7, -1, 3, -1, -1, -1, -1, -1, -1, -1]


@pytest.mark.parametrize("score", [route.SOFTMAX, route.SIGMOID])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_against_differences(score, renorm):
    rng = np.random.default_rng(2)
    z, dw = rng.normal(size=(3, 6)), rng.normal(size=(3, 2))
    ids, _, _ = route.choose(z, 2, score)

    def value(v):
        return (route.weights(route.scores(v, score)[1], ids, renorm, 1.5) * dw).sum()

    got = route.gradient(z, ids, dw, score, renorm, 1.5)
    step = 1e-6
    for t, e in itertools.product(range(3), range(6)):
        d = np.zeros_like(z)
        d[t, e] = step
        # central differences of a function with third derivatives of order 10: step^2 * 10 and 1e-16 / step of rounding
        assert abs((value(z + d) - value(z - d)) / (2 * step) - got[t, e]) < 2e-9


def test_quantize_by_hand():
    x = np.array([[127.0, -63.5, 0.5, 1.5], [0, 0, 0, 0], [1e-44, 0, 0, 0], [np.inf, 1, 1, 1], [1, np.nan, 1, 1]], np.float32)
    codes, scale = i8.quantize(x)
    assert codes[0].tolist() == [127, -64, 0, 2] and scale[0] == 1.0
    assert not codes[1].any() and scale[1] == 0.0
    assert codes[2].tolist() == [0, 0, 0, 0] and scale[2] == np.float32(2.0 ** -126)
    assert np.isnan(scale[3:]).all() and not codes[3:].any()


def test_quantize_half_step_bound():
    x = np.random.default_rng(3).normal(size=(50, 333)).astype(np.float32)
    codes, scale = i8.quantize(x)
    assert (np.abs(codes.astype(int)).max(-1) == 127).all()
    assert (np.abs(codes * scale[:, None].astype(np.float64) - x) <= scale[:, None] * (0.5 + 1e-4)).all()


def test_layout_and_product():
    rng = np.random.default_rng(4)
    a, b = rng.integers(-127, 128, (19, 80), dtype=np.int8), rng.integers(-127, 128, (16, 80), dtype=np.int8)
    flat = i8.layout(a).view(np.int8)
    assert flat.size == 32 * 128
    for r, k in itertools.product(range(19), range(80)):
        assert flat[((r // 16) * 2 + k // 64) * 1024 + (k % 64 // 16) * 256 + (r % 16) * 16 + k % 16] == a[r, k]
    one = np.ones(19, np.float32), np.full(16, 2.0, np.float32)
    want = np.array([[sum(int(x) * int(y) for x, y in zip(u, v)) for v in b] for u in a])
    assert np.array_equal(i8.matmul(a, one[0], b, one[1]), (2.0 * want).astype(np.float32))
