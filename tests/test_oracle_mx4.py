"""The oracle of 4-bit floating point and of the norm: codes by hand, the layout by its formula, gradients against differences."""
import numpy as np
import pytest

from oracle import mx4, norm


def test_codes_by_hand():
    x = np.zeros((1, 32), np.float32)
    x[0, :12] = [4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.26, 7.9, -0.0, 6]
    codes, scales = mx4.quantize(x)
    assert scales.tolist() == [[127]]
    assert codes[0, :12].tolist() == [6, 0, 2, 2, 4, 4, 6, 6, 9, 7, 8, 7]
    codes, scales = mx4.quantize(x, ceil=True)                # 7.9 > 6: a scale of 2
    assert scales.tolist() == [[128]] and codes[0, 9] == 6 and codes[0, 0] == 4


@pytest.mark.parametrize("top,floor,ceil", [(6.0, 127, 127), (6.0 * (1 + 2.0 ** -20), 127, 128), (4.0, 127, 127), (8.0, 128, 128), (2.0 ** -126, 0, 0),
                                            (1.5 * 2.0 ** -125, 0, 0), (2.0 ** -140, 0, 0), (3.4e38, 252, 252), (0.0, 0, 0)])
def test_scales(top, floor, ceil):
    x = np.zeros((1, 40), np.float32)
    x[0, 33] = -top
    assert mx4.quantize(x)[1].tolist() == [[0, floor]] and mx4.quantize(x, True)[1].tolist() == [[0, ceil]]


def test_no_number():
    x = np.ones((2, 64), np.float32)
    x[0, 5], x[1, 40] = np.nan, -np.inf
    codes, scales = mx4.quantize(x)
    assert scales.tolist() == [[255, 125], [125, 255]] and not codes[0, :32].any() and (codes[0, 32:] == 6).all()
    assert np.isnan(mx4.values(codes, scales)[0, :32]).all()


def test_error_is_half_a_step():
    x = np.random.default_rng(1).standard_normal((64, 96)).astype(np.float32)
    for ceil in (False, True):
        codes, scales = mx4.quantize(x, ceil)
        v = mx4.values(codes, scales)
        X = np.repeat(np.ldexp(1.0, scales.astype(int) - 127), 32, 1)
        a = np.abs(x) / X
        step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0)) * X
        inside = a <= 6
        assert (np.abs(v - x)[inside] <= step[inside] / 2).all() and (np.abs(v)[~inside] == 6 * X[~inside]).all()
        assert not ceil or inside.all()


def test_layout():
    rng = np.random.default_rng(2)
    codes, scales = rng.integers(0, 16, (20, 304), np.uint8), rng.integers(0, 250, (20, 10), np.uint8)
    c, s = mx4.layout(codes, scales)
    assert c.size == 32 * 256 and s.size == 32 * 16
    for r in (0, 7, 15, 16, 19):
        for k in (0, 1, 31, 32, 127, 128, 255, 256, 303):
            byte = c[((r // 16) * 4 + k // 128) * 1024 + k % 128 // 32 * 256 + r % 16 * 16 + k % 32 // 2]
            assert (byte >> 4 * (k % 2)) & 15 == codes[r, k]
            assert s[((r // 16) * 2 + k // 256) * 128 + (k % 128 // 32 * 16 + r % 16) * 2 + k % 256 // 128] == scales[r, k // 32]


def test_linear_gradients_against_differences():
    """Straight through the codes the layer is bilinear in what they stand for: central differences of it are exact but for rounding."""
    rng = np.random.default_rng(3)
    x, W, dy = rng.standard_normal((6, 32)), rng.standard_normal((16, 32)), rng.standard_normal((6, 16))
    Wt = mx4.quantize(W.T)
    xq, wq = mx4.values(*mx4.quantize(x.T)).T, mx4.values(*Wt).T
    dyc, dyr = mx4.values(*mx4.quantize(dy.T)).T, mx4.values(*mx4.quantize(dy))
    dx, dW = mx4.linear_bwd(dy, x, Wt)
    h = 0.5
    for i, j in ((0, 0), (5, 31), (2, 17)):
        e = np.zeros_like(x)
        e[i, j] = h
        assert abs((((x + e) @ wq.T - (x - e) @ wq.T) * dyr).sum() / (2 * h) - dx[i, j]) < 1e-12
    for i, j in ((0, 0), (15, 31), (7, 9)):
        e = np.zeros_like(W)
        e[i, j] = h
        assert abs(((xq @ (W + e).T - xq @ (W - e).T) * dyc).sum() / (2 * h) - dW[i, j]) < 1e-12


def test_norm_gradient_against_differences():
    rng = np.random.default_rng(4)
    s, g, dy, eps, h = rng.standard_normal((3, 48)), 1 + 0.1 * rng.standard_normal(48), rng.standard_normal((3, 48)), 1e-3, 1e-5
    _, rstd = norm.forward(s, g, eps)
    ds, dw = norm.backward(dy, s, rstd, g)
    for i, j in ((0, 0), (1, 20), (2, 47)):
        e = np.zeros_like(s)
        e[i, j] = h
        diff = ((norm.forward(s + e, g, eps)[0] - norm.forward(s - e, g, eps)[0]) * dy).sum() / (2 * h)
        assert abs(diff - ds[i, j]) < 1e-8                   # h^2 times a third derivative of order 1, and 2^-53 / h
    for j in (0, 20, 47):
        e = np.zeros_like(g)
        e[j] = h
        diff = ((norm.forward(s, g + e, eps)[0] - norm.forward(s, g - e, eps)[0]) * dy).sum() / (2 * h)
        assert abs(diff - dw[j]) < 1e-8
