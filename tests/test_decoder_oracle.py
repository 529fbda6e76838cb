"""CPU pins of the 4-bit decoder operators' oracle: codes against the format's own table and exhaustive search, scales against their definition."""
import numpy as np
import pytest

from oracle import decoder_oracle as O


def test_levels_are_the_formats():
    for c in range(16):
        e, m = (c >> 1) & 3, c & 1
        v = m * 0.5 if e == 0 else (1 + m / 2) * 2.0 ** (e - 1)
        assert O.e2m1_value(np.uint8(c)) == (-v if c & 8 else v)
    assert np.signbit(O.e2m1_value(np.array([8], np.uint8)))[0]


def test_codes_nearest_ties_even_saturating():
    x = np.array([0.0, 0.25, 0.2500001, 0.5, 0.75, 1.0, 1.25, 1.75, 2.5, 2.51, 3.5, 5.0, 5.01, 6.0, 7.0, 100.0, -0.75, -0.1, -9.0])
    assert O.e2m1_code(x).tolist() == [0, 0, 1, 1, 2, 2, 2, 4, 4, 5, 6, 6, 7, 7, 7, 7, 10, 8, 15]
    y = np.random.default_rng(3).uniform(-6.9, 6.9, 4000)
    got = O.e2m1_value(O.e2m1_code(y))
    every = np.concatenate([O.LEVELS, -O.LEVELS])
    assert np.array_equal(np.abs(got - y), np.abs(every[None, :] - y[:, None]).min(1))


@pytest.mark.parametrize("most,e", [(7.0, 0), (7.03125, 1), (3.5, -1), (3.515625, 0), (1.75, -2), (448.0, 6), (0.0, -120), (2.0 ** -130, -120), (6.0, 0)])
def test_group_exponent(most, e):
    x = np.zeros((1, 32))
    x[0, 5] = -most
    assert O.group_exponent(x)[0] == e


def test_values_of_a_vector():
    v = np.array([[6.0, -3.0, 0.6, 0.0]])
    code, s, w = O.quantise_vectors(v)
    assert s[0, 0] == 1.0 and w.tolist() == [[6.0, -3.0, 0.5, 0.0]]
    assert O.quantise_vectors(np.zeros((1, 4)))[1][0, 0] == 2.0 ** -120
    assert O.bf16(1.00390625) == 1.0 and O.bf16(1.01171875) == 1.015625


def test_attention_of_equal_values_and_empty_rows():
    rng = np.random.default_rng(1)
    q, k = rng.normal(size=(3, 4, 8)), rng.normal(size=(5, 2, 8))
    v = np.ones((5, 2, 8)) * 2.5
    out, spread, _ = O.attention(q, k, v, 0.3, [0, 2, 9])
    assert np.all(out[0] == 0) and np.allclose(out[1:], 2.5) and np.allclose(spread[1:], 2.5)
    one, _, _ = O.attention(q, k, rng.normal(size=(5, 2, 8)), 0.3, [1, 1, 1])
    assert np.allclose(one[:, 0], one[:, 1]) and not np.allclose(one[:, 0], one[:, 2])   # heads of a group share their kv head


def test_norm_of_a_constant_row():
    h, y = O.rmsnorm_residual(np.full((1, 16), 3.0), np.full((1, 16), -1.0), np.full(16, 0.5), 0.0)
    assert np.all(h == 2.0) and np.allclose(y, 0.5)
