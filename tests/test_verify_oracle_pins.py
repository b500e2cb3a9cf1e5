"""The oracle of the verification against cases worked out by hand."""
import numpy as np

from oracle.verify_oracle import draw, verify


def test_draws():
    r = np.array([0.0, 0.25, 0.0, 0.5, 0.25, 0.0])
    assert [draw(r, u) for u in (0.0, 0.2499, 0.25, 0.74, 0.75, 0.999, 1.0, 2.0, -1.0)] == [1, 1, 3, 3, 4, 4, 4, 4, 1]
    assert draw(np.zeros(3), 0.5) == -1


def test_chain():
    p = np.array([[0.5, 0.25, 0.25], [0.125, 0.875, 0.0], [0.0, 0.0, 1.0]])
    q = np.array([[0.25, 0.5, 0.25], [0.25, 0.25, 0.5], [1.0, 0.0, 0.0]])
    # token 1 after place 0: u * 0.5 < 0.25 where u < 0.5
    assert verify(p, q, [0, 1, 1], None, [0.5, 0.49, 0.0]) == ([0, 1, 2], 2)
    # refused at the border: what is left is max(p - q, 0) = (0.25, 0, 0)
    assert verify(p, q, [0, 1, 1], None, [0.9, 0.5, 0.0]) == ([0], 0)
    # the second one is token 0: u * 0.25 < 0.125; refused: left is (0, 0.625, 0)
    assert verify(p, q, [0, 1, 0], None, [0.3, 0.0, 0.5]) == ([0, 1], 1)


def test_siblings():
    p = np.array([[0.5, 0.25, 0.125, 0.125]] * 3)
    # picked tokens 1 and 0: refused with u >= 0.25, then 0.75 is left of which token 0 has 0.5: u * 0.75 < 0.5
    assert verify(p, None, [0, 1, 0], [-1, 0, 0], [0.1, 0.25, 0.6]) == ([0, 2], 0)
    assert verify(p, None, [0, 1, 0], [-1, 0, 0], [0.1, 0.25, 0.7]) == ([0], 2)
    # drawn ones: left is max(p - q, 0) = (0.25, 0, 0, 0), then m = 0.25
    q = np.array([[0.25] * 4] * 3)
    assert verify(p, q, [0, 2, 0], [-1, 0, 0], [0.1, 0.5, 0.99]) == ([0, 2], 0)
    # nothing is left of p: it is drawn from itself
    assert verify(p[:2], p[:2], [0, 2], [-1, 0], [0.6, 1.5]) == ([0], 1)
