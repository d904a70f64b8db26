"""Pins of the oracle's rotary positions and 8-bit cache (oracle/positions.py, oracle/cache.py): closed forms and brute force."""
import math

import numpy as np
import pytest

from oracle import cache, exact, fp8, positions


@pytest.mark.parametrize("interleaved", (False, True))
def test_rotation_is_a_rotation_of_each_pair(interleaved):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((2, 3, 5, 16))
    pos = rng.integers(-100, 100, (2, 5))
    f, m = positions.frequencies(12)
    y = positions.rotate(x, pos, f, interleaved, 1.0)
    u, v = positions.pairs(12, interleaved)
    assert m == 1.0 and sorted(np.concatenate((u, v)).tolist()) == list(range(12))
    for i in range(6):
        z = (x[..., u[i]] + 1j * x[..., v[i]]) * np.exp(1j * pos[:, None, :] * f[i])
        assert np.allclose(y[..., u[i]], z.real) and np.allclose(y[..., v[i]], z.imag)
    assert np.array_equal(y[..., 12:], x[..., 12:])
    assert np.allclose(positions.rotate(y, pos, f, interleaved, 1.0, inverse=True), x)
    # what it is for: the product of a rotated query and key depends on the distance alone
    a, b = x[:1, :1, :1, :12], x[1:, 1:2, 1:2, :12]
    dot = lambda p, q: float((positions.rotate(a, [[p]], f, interleaved) * positions.rotate(b, [[q]], f, interleaved)).sum())
    assert math.isclose(dot(7, 3), dot(1007, 1003), rel_tol=1e-9)


def test_scaled_frequencies():
    plain, _ = positions.frequencies(64)
    linear, _ = positions.frequencies(64, scaling="linear", factor=8.0)
    assert np.allclose(linear, plain / 8)
    ntk, _ = positions.frequencies(64, scaling="ntk", factor=8.0)
    assert math.isclose(ntk[0], 1.0) and math.isclose(ntk[-1], plain[-1] / 8)
    yarn, m = positions.frequencies(64, scaling="yarn", factor=8.0, original_length=4096)
    assert math.isclose(yarn[0], 1.0) and math.isclose(yarn[-1], plain[-1] / 8) and math.isclose(m, 1 + 0.1 * math.log(8))
    assert np.all(np.diff(yarn) < 0) and np.all(yarn <= plain + 1e-18) and np.all(yarn >= plain / 8 - 1e-18)


def test_exponents_and_codes():
    for amax in (0.0, 1e-40, 2.0 ** -100, 1.0, 447.9, 448.0, 448.0001, 1e30, 3e38):
        e = cache.exponent_for(amax)
        assert amax <= 448 * 2.0 ** e or e == cache.HIGHEST
        assert e == cache.LOWEST or amax > 448 * 2.0 ** (e - 1)
    assert cache.quantise([np.inf, -np.inf, 500.0, np.nan], 0)[:3].tolist() == [448.0, -448.0, 448.0]
    values = fp8.decode_all()
    values = values[np.isfinite(values)]
    assert np.array_equal(cache.quantise(values, 0), values)


def test_append_in_pieces_ends_where_append_at_once_does_when_scales_do_not_shrink_codes():
    """Growing scales only re-round codes that leave the normal range: with magnitudes in [1, 4) none does."""
    rng = np.random.default_rng(2)
    x = np.sign(rng.standard_normal((150, 8))) * (1 + 3 * rng.random((150, 8)))
    one, many = cache.Cache(192, 8), cache.Cache(192, 8)
    one.append(150, x, -x)
    at = 0
    for n in (1, 5, 70, 0, 64, 10):
        at += n
        many.append(at, x[at - n:at], -x[at - n:at])
    for w in range(2):
        assert np.array_equal(one.dequantised(w, 150), many.dequantised(w, 150))
        assert np.abs(one.dequantised(w, 150) - (x, -x)[w]).max() <= 4 * 2.0 ** -4


def test_attention_and_weights_against_the_plain_definition():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((5, 8)), rng.standard_normal((9, 8)), rng.standard_normal((9, 8))
    O, lse, size = cache.attend(q, k, v, 0.3, True)
    for i in range(5):
        s = 0.3 * k[:9 - 5 + i + 1] @ q[i]
        p = np.exp(s) / np.exp(s).sum()
        assert np.allclose(O[i], p @ v[:len(s)]) and np.isclose(lse[i], np.log(np.exp(s).sum()))
        assert np.allclose(size[i], p @ np.abs(v[:len(s)]))
    full = exact.forward(q, k, v, 0.3, False)
    assert np.allclose(cache.attend(q, k, v, 0.3, False)[0], full[0])
    w = cache.weights(q, k, lse, 0.3, True)
    assert math.isclose(w.sum(), 5.0) and w[8] < 1.0
    # rows that see nothing
    O, lse, _ = cache.attend(q, k[:3], v[:3], 0.3, True)
    assert (O[:2] == 0).all() and np.isneginf(lse[:2]).all() and np.isfinite(lse[2:]).all()
    assert math.isclose(cache.weights(q, k[:3], lse, 0.3, True).sum(), 3.0)


def test_kept_tokens():
    assert cache.kept([3.0, 1.0, 2.0], 3, 3, 1) == [0, 1, 2]
    assert cache.kept([3.0, 1.0, 2.0, 9.0], 4, 3, 1) == [0, 2, 3]
    assert cache.kept([1.0, 1.0, 1.0, 1.0, 0.0], 5, 3, 1) == [0, 1, 4]
    assert cache.kept([1.0, float("nan"), 5.0, 0.0], 4, 2, 0) == [1, 2]
    assert cache.kept([-0.0, 0.0, -1.0], 3, 1, 0) == [0]
    assert cache.kept([9.0, 8.0, 7.0], 3, 2, 2) == [1, 2]
