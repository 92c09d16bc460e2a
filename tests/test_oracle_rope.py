"""The rotation oracle against values worked by hand."""
import numpy as np

from oracle.rope import norm_rope


def test_quarter_turn_by_hand():
    x = np.zeros((1, 1, 8))
    x[0, 0] = [1, 2, 3, 4, 5, 6, 7, 8]
    f = np.array([np.pi / 2, 0.0])                       # pair 0 by a quarter turn at position 1, pair 1 not at all
    y, size = norm_rope(x, [1], f)                       # pairs (0, 2) and (1, 3), the rest as it was
    assert np.allclose(y[0, 0], [-3, 2, 1, 4, 5, 6, 7, 8])
    assert np.array_equal(size[0, 0], [4, 6, 4, 6, 5, 6, 7, 8])
    y, _ = norm_rope(x, [1], f, interleaved=True)        # pairs (0, 1) and (2, 3)
    assert np.allclose(y[0, 0], [-2, 1, 3, 4, 5, 6, 7, 8])


def test_norm_by_hand():
    x = np.array([[[3.0, -4.0, 0.0, 0.0]]])              # mean square 6.25
    y, _ = norm_rope(x, None, None, norm=True, weight=[1, 2, 3, 4], eps=0.0)
    assert np.allclose(y[0, 0], [1.2, -3.2, 0, 0])
    y, _ = norm_rope(x * 0, None, None, norm=True, eps=1e-6)
    assert (y == 0).all()


def test_products_of_rotated_rows_depend_on_the_distance_alone():
    r = np.random.default_rng(0)
    q, k = r.standard_normal((2, 1, 1, 128))
    f = 10000.0 ** (-np.arange(64) / 64)
    dots = [float((norm_rope(q, [p + 9], f)[0] * norm_rope(k, [p], f)[0]).sum()) for p in (0, 5, 4000)]
    assert np.allclose(dots, dots[0], atol=1e-9)
