"""The oracle of the cache in 4 bits against values worked out by hand, and the tests' quick packing against it."""
import numpy as np
import pytest

from oracle import kv4_oracle as o4
from tests import kv4_util


@pytest.mark.parametrize("a,x", [(0.0, -100), (6.0, 0), (6.0001, 1), (3.0, -1), (1.5, -2), (1.6, -1), (2.0 ** -120, -100), (3.3e38, 125), (6 * 2.0 ** 125, 125), (12.0, 1)])
def test_exponents(a, x):
    assert o4.exponent(a) == x


def test_nearest_code_ties_to_even():
    f = np.zeros(32)
    f[:16] = [6, 0.25, 0.26, 0.75, 0.74, 1.25, 1.75, 2.5, 2.51, 3.5, 5, 5.1, -0.25, -5, -0.75, -0.0]
    codes, x = o4.group(f)
    assert x == 0
    assert list(codes[:16]) == [7, 0, 1, 2, 1, 2, 4, 4, 5, 6, 6, 7, 8, 14, 10, 8]


def test_numbers():
    c, e = np.zeros((1, 32), np.int64), np.array([[3]])
    c[0, :4] = [7, 15, 1, 9]
    assert list(o4.numbers(c, e)[0, :4]) == [48, -48, 4, -4]
    assert np.isnan(o4.numbers(c, np.array([[-128]]))).all()


@pytest.mark.parametrize("dim,page", [(32, 32), (96, 64), (160, 128)])
def test_layout_by_hand_and_quick_packing(dim, page):
    rng = np.random.RandomState(0)
    a, b = o4.Pool(3, 2, dim, page, fill=5), o4.Pool(3, 2, dim, page, fill=5)
    pages, rows = np.array([1, 1, 2, 0]), np.array([0, 17, page - 1, 8])
    c = kv4_util.codes_of(rng, 4, 2, dim)
    kv4_util.place(b, pages, rows, *c)
    for i in range(4):
        a.write(pages[i], rows[i], [t[i] for t in c])
    for name in ("k", "v", "k_exp", "v_exp"):
        assert np.array_equal(getattr(a, name), getattr(b, name)), name
    for i in range(4):
        assert all(np.array_equal(x, y[i]) for x, y in zip(a.read(pages[i], rows[i]), c))
    # channel 16 f + n of row 32 b + 8 g + 2 j + half
    assert o4.value_byte(17, 18) == ((0, 2, 2, 1, 0), 1)
