"""Pins of the 4-bit cache's oracle: hand-worked codes, and properties that any right rounding has."""
import numpy as np
import pytest

import oracle.q4_oracle as Q


def test_codes_by_hand():
    # between neighbours: nearest, ties to the even code
    y = [0.0, 0.25, 0.26, 0.74, 0.75, 1.25, 1.26, 1.75, 2.5, 2.51, 3.49, 3.5, 5.0, 5.01, 6.0, 7.0, -0.25, -0.75, -7.0]
    assert Q.e2m1_round(y).tolist() == [0, 0, 1, 1, 2, 2, 3, 4, 4, 5, 5, 6, 6, 7, 7, 7, 0, 2, 7]


@pytest.mark.parametrize("top,e", [(0.0, -100), (7.0, 0), (7.0001, 1), (3.5, -1), (3.5001, 0), (6.0, 0), (4.0, 0), (1.0, -2),
                                   (448.0, 6), (1e-40, -100), (7.0 * 2.0 ** 112, 112), (np.inf, 112)])
def test_exponent_by_hand(top, e):
    assert Q.group_exponent(top) == e


def test_row_by_hand():
    x = np.zeros((1, 64))
    x[0, :4] = [7.0, -3.0, 0.75, -0.2]   # e = 0: 6, -3, 1, -0
    x[0, 33] = 0.0625                    # e = -6 (7 / 64 is above, 3.5 / 64 below): 4
    code, scale = Q.encode_rows(x)
    assert scale.tolist() == [[127, 121]]
    assert code[0, :2].tolist() == [0xd7, 0x82] and code[0, 16] == 0x60
    assert Q.decode_rows(code, scale)[0, [0, 1, 2, 3, 32, 33]].tolist() == [6.0, -3.0, 1.0, 0.0, 0.0, 0.0625]


def test_half_a_step():
    """No code is off by more than half the step at its place, and the exponent cannot be smaller."""
    g = np.random.default_rng(1)
    x = g.standard_normal((200, 64)) * 2.0 ** g.integers(-40, 40, (200, 1))
    code, scale = Q.encode_rows(x)
    v, unit = Q.decode_rows(code, scale), np.repeat(2.0 ** (scale.astype(float) - 127), 32, axis=1)
    a = np.abs(x) / unit
    step = np.where(a >= 4, 2.0, np.where(a >= 2, 1.0, 0.5))
    assert (np.abs(v - x) / unit <= step / 2).all()
    assert (np.abs(x).reshape(200, 2, 32).max(2) > 3.5 * 2.0 ** (scale.astype(float) - 127)).all()


def test_twice_is_once():
    g = np.random.default_rng(2)
    code, scale = Q.encode_rows(g.standard_normal((20, 128)))
    v = Q.decode_rows(code, scale)
    assert np.array_equal(Q.decode_rows(*Q.encode_rows(v)), v)


def test_nan_and_infinity():
    x = np.ones((1, 64))
    x[0, 3], x[0, 40] = np.nan, -np.inf
    v = Q.decode_rows(*Q.encode_rows(x))
    assert np.isnan(v[0, :32]).all() and v[0, 40] == -6 * 2.0 ** 112 and (np.delete(v[0, 32:], 8) == 0).all()


def test_weights_by_hand():
    # one query of zeros over two keys: half each; a query without keys adds nothing
    assert Q.key_weights(np.zeros((2, 4)), np.ones((2, 4)), [np.log(2.0), -np.inf], 0.5).tolist() == [0.5, 0.5]
    g = np.random.default_rng(3)
    q, k = g.standard_normal((7, 8)), g.standard_normal((11, 8))
    lse = np.log(np.exp(q @ k.T).sum(1))
    assert abs(Q.key_weights(q, k, lse, 1.0).sum() - 7) < 1e-12  # every query gives one in all


@pytest.mark.parametrize("w,keep,first,last,want", [
    ([1, 2, 3, 4, 5], 5, 0, 0, [0, 1, 2, 3, 4]), ([1, 2, 3, 4, 5], 7, 3, 3, [0, 1, 2, 3, 4]), ([5, 4, 3, 2, 1], 2, 0, 0, [0, 1]),
    ([1, 9, 2, 9, 1], 3, 1, 1, [0, 1, 4]), ([0, 0, 0, 0, 0, 0], 4, 1, 1, [0, 1, 2, 5]), ([3, 1, np.nan, 2], 2, 0, 0, [0, 2]),
    ([1, -1, -2, np.inf], 2, 0, 0, [0, 3]), ([9, 9, 9, 1, 2], 2, 0, 2, [3, 4]), ([1, 2, 9, 9], 2, 2, 0, [0, 1])])
def test_kept_by_hand(w, keep, first, last, want):
    assert Q.kept_tokens(np.array(w, dtype=float), keep, first, last) == want
