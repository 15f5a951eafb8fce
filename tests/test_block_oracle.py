"""Pins of the block's oracle: gradients against differences, closed forms, the packed layout against its declaration."""
import numpy as np
import pytest

from oracle import block_oracle as bo

RNG = np.random.default_rng(77)


def differences(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        g[i] = (f(up) - f(down)) / (2 * h)
    return g


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("masked", [False, True])
def test_gated_ff_gradients_are_differences(act, masked):
    X, Wg, Wu, dH = RNG.standard_normal((3, 4)), RNG.standard_normal((4, 5)), RNG.standard_normal((4, 5)), RNG.standard_normal((3, 5))
    mask = np.array([1, 0, 1, 1, 0]) if masked else None
    f = lambda x, a, b: float((bo.gated_ff(x, a, b, act, mask)[0] * dH).sum())  # noqa: E731
    dX, dWg, dWu, _, _ = bo.gated_ff_backward(dH, X, Wg, Wu, act, mask)
    # central differences in 64 bits: h^2 and 1e-16 / h, both below 1e-9 of the curvature here
    np.testing.assert_allclose(dX, differences(lambda v: f(v, Wg, Wu), X), rtol=1e-6, atol=1e-7)
    np.testing.assert_allclose(dWg, differences(lambda v: f(X, v, Wu), Wg), rtol=1e-6, atol=1e-7)
    np.testing.assert_allclose(dWu, differences(lambda v: f(X, Wg, v), Wu), rtol=1e-6, atol=1e-7)
    if masked:
        assert not dWg[:, mask == 0].any() and not dWu[:, mask == 0].any()


def test_gradients_from_saved_values_are_the_same():
    X, Wg, Wu, dH = RNG.standard_normal((3, 4)), RNG.standard_normal((4, 5)), RNG.standard_normal((4, 5)), RNG.standard_normal((3, 5))
    _, G, U = bo.gated_ff(X, Wg, Wu, "silu")
    for a, b in zip(bo.gated_ff_backward(dH, X, Wg, Wu, "silu"), bo.gated_ff_backward(dH, X, Wg, Wu, "silu", None, G, U)):
        np.testing.assert_array_equal(a, b)


def test_activations_in_closed_form():
    g = np.array([-50.0, -1.0, 0.0, 1.0, 50.0])
    np.testing.assert_allclose(bo.activation("silu", g), g / (1 + np.exp(-g)), atol=1e-15)
    np.testing.assert_allclose(bo.activation("gelu", np.array([1.0]))[0], 0.8413447460685429, rtol=1e-14)
    np.testing.assert_array_equal(bo.activation("relu", g), [0, 0, 0, 1, 50])
    np.testing.assert_allclose(bo.activation_slope("silu", np.zeros(1)), 0.5)
    np.testing.assert_allclose(bo.activation_slope("gelu", np.zeros(1)), 0.5)


@pytest.mark.parametrize("token_gate", [False, True])
def test_block_norm_gradients_are_differences(token_gate):
    t, n = 3, 4
    x, b, dr, dy = (RNG.standard_normal((t, n)) for _ in range(4))
    wp, wq = RNG.standard_normal(n), RNG.standard_normal(n)
    gate = RNG.standard_normal((t, n) if token_gate else n)
    eps, scale = 1e-2, 0.7

    def f(x, b, wp, gate, wq):
        r, y = bo.block_norm(x, b, wp, gate, wq, scale, eps)
        return float((r * dr).sum() + (y * dy).sum())

    r, _ = bo.block_norm(x, b, wp, gate, wq, scale, eps)
    dx, db, dwp, dg, dwq = bo.block_norm_backward(dr, dy, r, b, wp, gate, wq, scale, eps)
    tol = dict(rtol=1e-6, atol=1e-7)
    np.testing.assert_allclose(dx, differences(lambda v: f(v, b, wp, gate, wq), x), **tol)
    np.testing.assert_allclose(db, differences(lambda v: f(x, v, wp, gate, wq), b), **tol)
    np.testing.assert_allclose(dwp, differences(lambda v: f(x, b, v, gate, wq), wp), **tol)
    np.testing.assert_allclose(dg, differences(lambda v: f(x, b, wp, v, wq), gate), **tol)
    np.testing.assert_allclose(dwq, differences(lambda v: f(x, b, wp, gate, v), wq), **tol)


def test_a_normed_row_has_unit_mean_square():
    x = RNG.standard_normal((5, 300)) * 10
    _, y = bo.block_norm(x, w_pre=np.ones(300), eps=0.0)
    np.testing.assert_allclose((y * y).mean(1), 1.0, rtol=1e-14)


def test_quantising_is_the_nearest_value_and_exact_on_the_grid():
    grid = np.concatenate([bo.E2M1, -bo.E2M1[1:], [0.0]]).astype(np.float32)[:, None]      # 16 rows, largest 6: scale 1
    codes, scales = bo.w4_quantise(grid, 32)
    assert scales[0, 0] == 1.0
    np.testing.assert_array_equal(bo.w4_values(codes, scales, 32), grid)
    W = RNG.standard_normal((200, 7)).astype(np.float32)
    W[:, 3] = 0
    codes, scales = bo.w4_quantise(W, 64)
    V = bo.w4_values(codes, scales, 64)
    steps = np.repeat(scales, 64, axis=0)[:200]
    # no value of the grid is nearer than the chosen one
    every = np.concatenate([bo.E2M1, -bo.E2M1])[:, None, None] * steps[None]
    np.testing.assert_allclose(np.abs(V - W), np.abs(every - W[None]).min(0), rtol=1e-6, atol=1e-12)
    assert not V[:, 3].any() and not scales[:, 3].any()
    # ties go to the smaller magnitude
    tie = np.array([[6.0], [2.5], [0.25], [-5.0], [1.25]], np.float32)
    np.testing.assert_array_equal(bo.w4_values(*bo.w4_quantise(tie, 32), 32)[:, 0], [6, 2, 0, -4, 1])


def test_bf16_rounding_of_scales():
    import torch
    x = RNG.standard_normal(4000).astype(np.float32)
    np.testing.assert_array_equal(bo.to_bf16(x), torch.from_numpy(x).bfloat16().float().numpy())


def test_packed_layout():
    W = RNG.standard_normal((130, 18)).astype(np.float32)
    codes, scales = bo.w4_quantise(W, 32)
    packed, laid = bo.w4_layout(codes, scales, 32)
    assert packed.shape == (2, 2, 64, 16) and laid.shape == (2, 2, 16, 4)
    # entry l, byte 4 q + i: column l % 16, rows 32 q + 8 (l / 16) + 2 i (low half) and the next one
    assert packed[1, 0, 17, 4 * 2 + 3] & 15 == codes[64 + 8 + 6, 17]
    assert packed[1, 0, 17, 4 * 2 + 3] >> 4 == codes[64 + 8 + 7, 17]
    assert laid[1, 0, 1, 2] == scales[2, 17]
    assert not packed[1, :, 2::16].any() and not laid[1, :, 2:].any(), "past the matrix"
