"""Pins of the oracle's rotary positions: a hand-worked vector, complex
multiplication, invariants (norms, relative positions, axes), and the append's
slots and fp8 range."""
import numpy as np
import pytest

from oracle import kap_oracle as O


def test_worked_vector():
    # one head of 4 dims, frequencies 1 and 1/2 quarter turns per position
    f = np.array([np.pi / 2, np.pi / 4])
    x = np.array([[[1.0, 2.0, 3.0, 4.0]]])
    r = np.sqrt(0.5)
    # position 1: dims (0, 2) by 90 degrees, dims (1, 3) by 45
    assert np.allclose(O.rotate(x, [1], f), [[[-3.0, (2 - 4) * r, 1.0, (4 + 2) * r]]])
    # pairs: dims (0, 1) by 90 degrees, dims (2, 3) by 45
    assert np.allclose(O.rotate(x, [1], f, pairs=True), [[[-2.0, 1.0, (3 - 4) * r, (4 + 3) * r]]])
    # the second frequency on the second axis, whose position is 2: 90 degrees
    assert np.allclose(O.rotate(x, [[1], [2]], f, [0, 1]), [[[-3.0, -4.0, 1.0, 2.0]]])
    # an axis that does not exist turns nothing
    assert np.allclose(O.rotate(x, [1], f, [0, 7]), [[[-3.0, 2.0, 1.0, 4.0]]])


@pytest.mark.parametrize("pairs", [False, True])
def test_against_complex_numbers(pairs):
    rng = np.random.default_rng(1)
    T, H, D, n = 7, 3, 20, 8                      # 16 of 20 dims turned
    x = rng.standard_normal((T, H, D))
    pos, axis = rng.integers(-5, 300000, (3, T)), rng.integers(0, 3, n)
    f = 1e4 ** (-np.arange(n) / n)
    z = x[..., 0:16:2] + 1j * x[..., 1:16:2] if pairs else x[..., :8] + 1j * x[..., 8:16]
    z = z * np.exp(1j * (pos[axis].T * f))[:, None, :]
    got = O.rotate(x, pos, f, axis, pairs)
    assert np.allclose(got[..., 0:16:2] if pairs else got[..., :8], z.real, atol=1e-12)
    assert np.allclose(got[..., 1:16:2] if pairs else got[..., 8:16], z.imag, atol=1e-12)
    assert np.array_equal(got[..., 16:], x[..., 16:])


def test_products_depend_on_the_distance_alone():
    rng = np.random.default_rng(2)
    q, k = rng.standard_normal((1, 1, 32)), rng.standard_normal((1, 1, 32))
    f = 1e3 ** (-np.arange(16) / 16)
    at = lambda m, n: float(np.sum(O.rotate(q, [m], f) * O.rotate(k, [n], f)))
    assert abs(at(17, 5) - at(1012, 1000)) < 1e-9
    assert abs(at(5, 5) - float(np.sum(q * k))) < 1e-12


def test_append_places_and_limits():
    P, Hkv, D = 3, 2, 64
    scales = np.array([[1.0, 1.0], [0.5, 0.25], [2.0, 0.0625]], np.float32)
    pool = O.KVPool(np.zeros((P, Hkv, D // 8, 16, 8), np.uint8), np.zeros((P, Hkv, D, 16), np.uint8),
                    "fp8", scales)
    rng = np.random.default_rng(3)
    k, v = rng.standard_normal((4, Hkv, D)), 40 * rng.standard_normal((4, Hkv, D))
    slots, pos = [16 + 3, -1, 47, 48], [9, 8, 7, 6]
    f = np.array([0.3, 0.2, 0.1, 0.05, 0.02, 0.01, 0.005, 0.001])
    q, kp, vp, bad = O.rope_append_kv(pool, None, k, v, slots, pos, f)
    assert q is None and bad == 1
    turned = O.rotate(k, pos, f)
    assert np.allclose(kp[1, :, :, 3].reshape(Hkv, D), turned[0] / 0.5)
    assert np.allclose(kp[2, :, :, 15].reshape(Hkv, D), turned[2] / 2.0)
    assert np.allclose(vp[2, :, :, 15], np.clip(v[2] / 0.0625, -448, 448))
    assert np.abs(v[2] / 0.0625).max() > 448
    written = ~np.isnan(kp[:, 0, 0, :, 0])
    assert written.sum() == 2 and written[1, 3] and written[2, 15]
    assert np.array_equal(~np.isnan(vp[:, 0, 0, :]), written)


@pytest.mark.parametrize("pairs", [False, True])
def test_an_angle_of_zero_leaves_infinities_alone(pairs):
    inf = np.inf
    x = np.array([[[inf, 2.0, 3.0, -inf, 5.0, np.nan, 7.0, 8.0]]])
    f = np.array([0.1, 0.2, inf, 0.4])
    # position 0, and axes that do not exist
    assert np.array_equal(O.rotate(x, [0], f[:2], None, pairs), x, equal_nan=True)
    assert np.array_equal(O.rotate(x, [9], f, [1, -1, 7, 2], pairs), x, equal_nan=True)
    # the other frequencies turn their pairs
    some = O.rotate(x, [9], f, [1, 0, 7, 2], pairs)
    turned = [2, 3] if pairs else [1, 5]
    keep = [d for d in range(8) if d not in turned]
    assert np.array_equal(some[0, 0, keep], x[0, 0, keep], equal_nan=True)
    assert not np.array_equal(some[0, 0, turned], x[0, 0, turned], equal_nan=True)
