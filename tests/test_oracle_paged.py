"""Pins of the oracle's steps around a decode step: the position rotation, the log of
the attention's sum, and log probabilities with their entropy and order."""
import math

import numpy as np
import pytest

from oracle import ripple_oracle as O


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_by_known_angles(interleaved):
    # two pairs with angles pi/2 and pi at position 1: (x, y) -> (-y, x) and (-x, -y)
    x = np.array([[1.0, 2.0, 3.0, 4.0, 9.0]])
    got = O.rotate(x, [1], [math.pi / 2, math.pi], interleaved)
    want = [-2, 1, -3, -4, 9] if interleaved else [-3, -2, 1, -4, 9]
    np.testing.assert_allclose(got[0], want, atol=1e-15)
    np.testing.assert_array_equal(O.rotate(x, [0], [0.3, 2.0], interleaved), x)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotated_products_depend_on_the_distance_alone(interleaved):
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 16))
    inv = 10.0 ** -np.arange(8)
    dot = lambda a, b: (O.rotate(q, [a], inv, interleaved) @ O.rotate(k, [b], inv, interleaved).T).item()  # noqa: E731
    assert dot(7, 3) == pytest.approx(dot(104, 100), abs=1e-12)
    assert abs(dot(7, 3) - dot(8, 3)) > 1e-3
    # shapes with heads: the same as head by head
    x = rng.standard_normal((3, 2, 16))
    both = O.rotate(x, [1, 5, 9], inv, interleaved)
    for h in range(2):
        np.testing.assert_array_equal(both[:, h], O.rotate(x[:, h], [1, 5, 9], inv, interleaved))


def test_lse_joins_two_parts_of_a_cache():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((2, 8)), rng.standard_normal((9, 8)), rng.standard_normal((9, 8))
    a, b = slice(0, 4), slice(4, 9)
    la, lb, l = (O.attention_lse(q, k[s], 0.5) for s in (a, b, slice(0, 9)))
    np.testing.assert_allclose(np.logaddexp(la, lb), l, atol=1e-14)
    o = sum(np.exp(x - l)[:, None] * O.decode_attention(q, k[s], v[s], 0.5)
            for x, s in ((la, a), (lb, b)))
    np.testing.assert_allclose(o, O.decode_attention(q, k, v, 0.5), atol=1e-14)


def test_logprobs_closed_forms():
    lp, h = O.token_logprobs(np.zeros(7))
    np.testing.assert_allclose(lp, -math.log(7), atol=1e-15)
    assert h == pytest.approx(math.log(7))
    # one likely token among masked ones and n - 1 equal others at temperature 2
    x = np.array([4.0, 0.0, -np.inf, 0.0, 0.0])
    lp, h = O.token_logprobs(x, 0.5)
    p = math.exp(2) / (math.exp(2) + 3)
    assert lp[0] == pytest.approx(math.log(p)) and lp[2] == -np.inf
    assert h == pytest.approx(-p * math.log(p) - (1 - p) * math.log((1 - p) / 3))


def test_top_tokens_break_ties_by_index():
    x = np.array([1.0, 3.0, -np.inf, 3.0, 0.0, -0.0])
    assert O.top_tokens(x, 6).tolist() == [1, 3, 0, 4, 5, 2]
