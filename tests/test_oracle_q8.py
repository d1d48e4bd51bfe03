"""Pins of the 8-bit cache's oracle: the e4m3 grid, its rounding, block exponents, appends and rotations in closed form."""
import numpy as np
import pytest
import torch

import oracle as O


def test_grid_is_e4m3():
    g = O.e4m3_grid()
    assert len(g) == 127 and g[0] == 0 and g[1] == 2.0 ** -9 and g[8] == 2.0 ** -6 and g[-1] == 448.0
    assert (np.diff(g) > 0).all()
    # every byte as torch reads it
    b = torch.arange(256, dtype=torch.uint8)
    want = b.view(torch.float8_e4m3fn).float().numpy()
    got = O.codes_of_bytes(b.numpy())
    assert np.array_equal(np.isnan(want), np.isnan(got)) and np.array_equal(want[~np.isnan(want)], got[~np.isnan(got)])


def test_rounding_is_nearest_even():
    r = np.random.default_rng(1)
    y = np.concatenate([r.uniform(-448, 448, 4000), r.standard_normal(4000) * 2.0 ** -7, [0.0, 448.0, -448.0, 1e9, -1e9]])
    y = y.astype(np.float32).astype(np.float64)
    want = torch.from_numpy(np.clip(y, -448, 448)).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.e4m3_round(y), want)
    g = O.e4m3_grid()
    mid = (g[1:] + g[:-1]) / 2  # ties go to the even code
    assert np.array_equal(O.e4m3_round(mid), np.where(np.arange(126) % 2 == 0, g[:-1], g[1:]))
    assert np.isnan(O.e4m3_round(np.nan))


def test_block_exponent_closed_form():
    for e in (-40, -3, 0, 1, 7, 60):
        assert O.block_exponent(448.0 * 2.0 ** e) == e
        assert O.block_exponent(np.nextafter(448.0 * 2.0 ** e, np.inf)) == e + 1
    assert O.block_exponent(0.0) == O.E_MIN and O.block_exponent(1e-300) == O.E_MIN
    assert O.block_exponent(np.inf) == O.E_MAX


def test_append_in_steps_keeps_what_is_held():
    """A block filled in two appends: the first codes move to the larger scale, exactly but for subnormals."""
    G, d = 16, 4
    v, e = np.zeros((32, d)), np.zeros(2, dtype=int)
    O.append_codes(v, e, np.full((5, d), 3.0), 0, G)
    assert e[0] == O.block_exponent(3.0) == -7 and np.array_equal(O.cache_values(v, e, G)[:5], np.full((5, d), 3.0))
    O.append_codes(v, e, np.full((14, d), 100.0), 5, G)
    x = O.cache_values(v, e, G)
    assert e[0] == e[1] == O.block_exponent(100.0) == -2
    # 100 = 400 / 4 lies between the codes 384 and 416, a tie that goes to the even code, 384
    assert np.array_equal(x[:5], np.full((5, d), 3.0)) and np.array_equal(x[5:19], np.full((14, d), 96.0))


@pytest.mark.parametrize("layout", ["pairs", "halves"])
def test_rotation_keeps_lengths_and_turns_back(layout):
    r = np.random.default_rng(2)
    x, ang = r.standard_normal((7, 16)), r.uniform(0, 6, (7, 8))
    cs = np.stack([np.cos(ang), np.sin(ang)], 2)
    y = O.norm_rope(x, None, 0.0, None, cs, layout)
    assert np.allclose((y ** 2).sum(1), (x ** 2).sum(1), rtol=1e-12)
    back = O.norm_rope(y, None, 0.0, None, np.stack([np.cos(ang), -np.sin(ang)], 2), layout)
    assert np.allclose(back, x, atol=1e-12)
    quarter = np.zeros((7, 8, 2))
    quarter[..., 1] = 1.0  # a quarter turn: (a, b) -> (-b, a)
    y = O.norm_rope(x, None, 0.0, None, quarter, layout)
    a, b = (slice(0, None, 2), slice(1, None, 2)) if layout == "pairs" else (slice(0, 8), slice(8, 16))
    assert np.array_equal(y[:, a], -x[:, b]) and np.array_equal(y[:, b], x[:, a])


def test_norms_closed_form():
    x = np.array([[3.0, 4.0, 0.0, 0.0], [0.0] * 4])
    assert np.allclose(O.norm_rope(x, "l2", 1e-6, None, None, "pairs"), [[0.6, 0.8, 0, 0], [0] * 4])
    assert np.allclose(O.norm_rope(x[:1], "rms", 0.0, np.full(4, 2.0), None, "pairs")[0], [2.4, 3.2, 0, 0])
