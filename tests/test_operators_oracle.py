"""The operators' oracle against tables, hand-worked values and differences (CPU)."""

import numpy as np
import pytest

from oracle import operators as O


def test_every_code_and_its_neighbours():
    # one block per value under test: 6 fixes the scale at 1 (floor(log2 6) - 2 = 0)
    cases = [(0.0, 0), (0.24, 0), (0.25, 0), (0.26, 1), (0.5, 1), (0.74, 1), (0.75, 2), (1.0, 2), (1.25, 2), (1.26, 3),
             (1.5, 3), (1.75, 4), (2.0, 4), (2.5, 4), (2.51, 5), (3.0, 5), (3.5, 6), (4.0, 6), (5.0, 6), (5.01, 7), (6.0, 7),
             (7.9, 7)]
    for v, want in cases:
        x = np.zeros((1, 32))
        x[0, 0], x[0, 1], x[0, 2] = 6.0, v, -v
        codes, scales = O.mx_quantize(x)
        assert scales[0, 0] == 127 and codes[0, 0] == 7 | want << 4 and codes[0, 1] == want + 8, v


def test_scales():
    for v, want in [(1.0, 125), (1.99, 125), (4.0, 127), (2.0 ** 127, 252), (2.0 ** -124, 1), (2.0 ** -125, 0), (2.0 ** -133, 0),
                    (0.0, 0), (np.inf, 255), (np.nan, 255)]:
        _, scales = O.mx_quantize(np.full((1, 32), v))
        assert scales[0, 0] == want, v
    assert (O.mx_quantize(np.ones((2, 33)))[1] == [[125, 125, 0, 0]] * 2).all()


def test_values_survive_packing():
    rng = np.random.default_rng(0)
    codes = rng.integers(0, 256, (8, 64), dtype=np.uint8)
    codes[:, ::16] |= 7    # each block's first value is 6: the scale is found again
    scales = rng.integers(2, 250, (8, 4), dtype=np.uint8)
    v = O.mx_values(codes, scales, 128)
    c2, s2 = O.mx_quantize(v)
    np.testing.assert_array_equal(s2, scales)
    np.testing.assert_array_equal(O.mx_values(c2, s2, 128), v)


def test_route_by_hand():
    l = np.array([[0.0, 2.0, 2.0, 1.0], [-np.inf] * 4, [-np.inf, 5.0, -np.inf, -np.inf]])
    w, ids, counts, order = O.route(l, 2, True)
    np.testing.assert_array_equal(ids, [[1, 2], [-1, -1], [1, -1]])
    np.testing.assert_allclose(w, [[0.5, 0.5], [0, 0], [1, 0]])
    np.testing.assert_array_equal(counts, [0, 2, 1, 0])
    np.testing.assert_array_equal(order, [0, 4, 1, -1, -1, -1])


@pytest.mark.parametrize("normalize", [True, False])
def test_route_gradient_against_differences(normalize):
    rng = np.random.default_rng(1)
    l, g = rng.normal(size=(5, 7)) * 2, rng.normal(size=(5, 3))
    l[2, 4] = -np.inf
    _, ids, _, _ = O.route(l, 3, normalize)
    d = O.route_backward(l, ids, g, normalize)
    h = 1e-6
    for t in range(5):
        for e in range(7):
            if l[t, e] == -np.inf:
                assert d[t, e] == 0
                continue
            f = []
            for s in (h, -h):
                m = l.copy()
                m[t, e] += s
                w, i, _, _ = O.route(m, 3, normalize)
                assert (i == ids).all()
                f.append((w * g).sum())
            assert abs((f[0] - f[1]) / (2 * h) - d[t, e]) < 1e-8


def test_layer_by_hand():
    # one expert of inner size 1: y = Wd silu(Wg x) (Wu x)
    x = np.array([[2.0, -1.0]])
    up = np.array([[[1.0, 0.0], [0.0, 3.0]]])
    down = np.array([[[4.0], [-1.0]]])
    y, bound = O.moe_layer(x, np.zeros((1, 2)), up, down, 1, True)
    h = 2 / (1 + np.exp(-2.0)) * -3
    np.testing.assert_allclose(y, [[4 * h, -h]])
    assert (bound >= np.abs(y)).all()
