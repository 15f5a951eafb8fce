"""Pins of the oracle of the product with an epilogue, dropout and 8 bits: published vectors of the generator, gradients against
differences, the 8-bit format against an enumeration of its codes."""
import numpy as np
import pytest

from oracle import linear_oracle as lo

RNG = np.random.default_rng(78)


def test_generator_against_its_published_vectors():
    """The known answers that the authors of Philox distribute with it (Philox4x32, ten rounds)."""
    known = [((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
             ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
             ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))]
    for counter, key, words in known:
        assert tuple(lo.philox4x32(np.array(counter, dtype=object), key)) == words


def test_kept_shares_and_places():
    k = lo.kept(200, 500, 0.3, 12345678901234567890, 7)
    # 1e5 draws: five standard deviations of the share are 0.0073
    assert abs(k.mean() - 0.7) < 0.0073
    np.testing.assert_array_equal(lo.kept([3, 199], [0, 1, 5, 499], 0.3, 12345678901234567890, 7), k[np.ix_([3, 199], [0, 1, 5, 499])])
    assert (lo.kept(200, 500, 0.3, 12345678901234567890, 8) != k).mean() > 0.3
    assert lo.kept(4, 4, 0.0, 1).all()


@pytest.mark.parametrize("act", [None, "silu", "gelu", "relu"])
@pytest.mark.parametrize("drop", [None, (0.4, 11, 3)])
def test_linear_gradients_are_differences(act, drop):
    X, W, b, dY = RNG.standard_normal((3, 4)), RNG.standard_normal((4, 5)), RNG.standard_normal(5), RNG.standard_normal((3, 5))
    f = lambda X, W, b: float((lo.linear(X, W, b, 0.0, act, drop)[0] * dY).sum())  # noqa: E731
    Z = lo.linear(X, W, b, 0.0, act, drop)[1]
    got = lo.linear_backward(dY, X, W, Z, act, drop)
    h = 1e-6
    for k, v in enumerate((X, W, b)):
        at = [X, W, b]
        g = np.zeros_like(v)
        for i in np.ndindex(v.shape):
            up, down = v.copy(), v.copy()
            up[i] += h
            down[i] -= h
            g[i] = (f(*(at[:k] + [up] + at[k + 1:])) - f(*(at[:k] + [down] + at[k + 1:]))) / (2 * h)
        # central differences in 64 bits: h^2 and 1e-16 / h, both below 1e-9 of the curvature here
        np.testing.assert_allclose(got[k], g, rtol=1e-6, atol=1e-7)


def all_codes():
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (1 + m / 8) * 2.0 ** (e - 7.0), m / 8 * 2.0 ** -6)
    v = np.where((e == 15) & (m == 7), np.nan, v)
    return np.where(c > 127, -v, v)


def test_rounding_to_codes_is_nearest_and_ties_go_to_the_even_code():
    codes = all_codes()
    positive = codes[:127]                       # 0 .. 448 in order: a code's number is its place
    assert positive[-1] == 448 and (np.diff(positive) > 0).all()
    v = np.concatenate((positive, (positive[1:] + positive[:-1]) / 2, RNG.uniform(0, 448, 2000), RNG.uniform(0, 0.02, 2000)))
    for x, q in zip(v, lo.e4m3(v)):
        d = np.abs(positive - x)
        near = np.flatnonzero(d == d.min())
        assert q == positive[near[0] if len(near) == 1 else near[near % 2 == 0][0]]
    np.testing.assert_array_equal(lo.e4m3(-v), -lo.e4m3(v))


def test_scales_are_the_smallest_that_clip_nothing():
    top = np.concatenate((np.exp2(RNG.uniform(-120, 120, 500)), [448.0, 449.0, 447.0, 224.0, 225.0, 1.75, np.nextafter(1.75, 2)]))
    s = lo.e8m0(top)
    # (2^-127 is the smallest there is)
    assert (top <= 448 * s).all() and ((top > 448 * s / 2) | (s == 2.0 ** -127)).all()
    np.testing.assert_array_equal(lo.e8m0(np.array([0.0, 1e-45])), 2.0 ** -127)


def test_packing():
    A = RNG.standard_normal((3, 200)) * np.exp2(RNG.integers(-20, 20, (3, 200)))
    A[1, 40] = np.inf
    codes, s = lo.pack8(A)
    assert codes.shape == (3, 256) and s.shape == (3, 8)
    assert np.isnan(codes[1, 32:64]).all() and np.isfinite(codes).sum() == 3 * 256 - 32 and not codes[:, 200:].any()
    back = lo.unpack8(codes, s, 200)
    fine = np.isfinite(back)
    group = np.repeat(s, 32, 1)[:, :200]
    # half a step: 2^-4 of the value, or of the smallest normal code's binade
    assert (np.abs(back - A)[fine] <= np.maximum(np.abs(A) * 2.0 ** -4, group * 2.0 ** -10)[fine]).all()


def test_a_dropped_entry_s_gradient_is_zero_whatever_its_pre_activation_was():
    X, W, dY, Z = RNG.standard_normal((6, 4)), RNG.standard_normal((4, 8)), RNG.standard_normal((6, 8)), RNG.standard_normal((6, 8))
    drop = (0.5, 21, 2)
    want = lo.linear_backward(dY, X, W, Z, "silu", drop)
    Z[~lo.kept(6, 8, *drop)] = np.nan
    for p, q in zip(lo.linear_backward(dY, X, W, Z, "silu", drop), want):
        np.testing.assert_array_equal(p, q)
