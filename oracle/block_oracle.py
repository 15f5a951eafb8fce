"""Independent oracle of the pruned feed-forward block: every operator by its definition, in 64 bits, with
numpy and scipy on the CPU.  It shares no code with the HIP path.

Weights are n x m with the hidden channels as columns, tokens are rows."""
import numpy as np
from scipy import special


def activation(kind, g):
    if kind == "silu":
        return g * special.expit(g)
    if kind == "gelu":
        return g * special.ndtr(g)
    return np.maximum(g, 0.0)


def activation_slope(kind, g):
    if kind == "silu":
        s = special.expit(g)
        return s + g * s * (1 - s)
    if kind == "gelu":
        return special.ndtr(g) + g * np.exp(-0.5 * g * g) / np.sqrt(2 * np.pi)
    return (g > 0).astype(np.float64)


def gated_ff(X, Wg, Wu, act, mask=None):
    """H, G, U; pruned channels are zeros."""
    X, Wg, Wu = (np.asarray(a, np.float64) for a in (X, Wg, Wu))
    G, U = X @ Wg, X @ Wu
    H = activation(act, G) * U
    if mask is not None:
        pruned = np.asarray(mask) == 0
        H[:, pruned] = G[:, pruned] = U[:, pruned] = 0.0
    return H, G, U


def gated_ff_backward(dH, X, Wg, Wu, act, mask=None, G=None, U=None):
    """dX, dWg, dWu, and the gradients dG, dU they come from."""
    dH, X, Wg, Wu = (np.asarray(a, np.float64) for a in (dH, X, Wg, Wu))
    if G is None:
        G, U = X @ Wg, X @ Wu
    dG = dH * np.asarray(U, np.float64) * activation_slope(act, np.asarray(G, np.float64))
    dU = dH * activation(act, np.asarray(G, np.float64))
    if mask is not None:
        pruned = np.asarray(mask) == 0
        dG[:, pruned] = dU[:, pruned] = 0.0
        Wg, Wu = Wg.copy(), Wu.copy()
        Wg[:, pruned] = Wu[:, pruned] = 0.0
    return dG @ Wg.T + dU @ Wu.T, X.T @ dG, X.T @ dU, dG, dU


def rms(z, eps):
    return np.sqrt((z * z).mean(1, keepdims=True) + eps)


def block_norm(x, b=None, w_post=None, gate=None, w_pre=None, scale=1.0, eps=1e-6):
    """r, y."""
    x = np.asarray(x, np.float64)
    r = x
    if b is not None:
        b, w_post, gate = (np.asarray(a, np.float64) for a in (b, w_post, gate))
        r = x + scale * gate * (w_post * (b / rms(b, eps)))
    return r, None if w_pre is None else np.asarray(w_pre, np.float64) * (r / rms(r, eps))


def _rms_norm_backward(z, g, eps):
    """Gradient of <g, z / rms(z)> at z: (g - zh mean(zh g)) / rms with zh = z / rms(z)."""
    s = rms(z, eps)
    zh = z / s
    return (g - zh * (zh * g).mean(1, keepdims=True)) / s


def block_norm_backward(dr, dy, r, b=None, w_post=None, gate=None, w_pre=None, scale=1.0, eps=1e-6):
    """dx, db, dw_post, dgate (per entry of the gate as given), dw_pre."""
    r = np.asarray(r, np.float64)
    dx = np.zeros_like(r) if dr is None else np.asarray(dr, np.float64).copy()
    db = dw_post = dgate = dw_pre = None
    if w_pre is not None:
        dy = np.asarray(dy, np.float64)
        dx += _rms_norm_backward(r, np.asarray(w_pre, np.float64) * dy, eps)
        dw_pre = (dy * (r / rms(r, eps))).sum(0)
    if b is not None:
        b, w_post, gate = (np.asarray(a, np.float64) for a in (b, w_post, gate))
        bh = b / rms(b, eps)
        db = _rms_norm_backward(b, scale * gate * w_post * dx, eps)
        dw_post = (scale * gate * dx * bh).sum(0)
        dgate = scale * dx * w_post * bh
        if gate.ndim == 1:
            dgate = dgate.sum(0)
    return dx, db, dw_post, dgate, dw_pre


E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def to_bf16(x):
    """Round to bf16, nearest, ties to even; finite values."""
    bits = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    bits = (bits + 0x7fff + ((bits >> 16) & 1)) & 0xffff0000
    return bits.astype(np.uint32).view(np.float32)


def w4_quantise(W, group):
    """codes (n x m, 0..15) and scales (groups x m, bf16 values) of a matrix of fp32 values."""
    W = np.asarray(W, np.float32)
    n, m = W.shape
    groups = -(-n // group)
    codes, scales = np.zeros((n, m), np.uint8), np.zeros((groups, m), np.float32)
    for g in range(groups):
        rows = W[g * group:(g + 1) * group]
        scale = to_bf16(np.abs(rows).max(0) / np.float32(6))
        scales[g] = scale
        v = np.abs(rows) / np.where(scale > 0, scale, np.float32(1))
        v[:, scale == 0] = 0
        # the nearest value, the smaller one of two equally near
        nearest = np.abs(v[..., None].astype(np.float64) - E2M1).argmin(-1)
        codes[g * group:(g + 1) * group] = nearest + 8 * (rows < 0)
    return codes, scales


def w4_values(codes, scales, group):
    value = np.where(codes >= 8, -E2M1[codes & 7], E2M1[codes & 7])
    return value * np.repeat(scales.astype(np.float64), group, axis=0)[:codes.shape[0]]


def w4_layout(codes, scales, group):
    """The packed form, entry by entry: uint8 [column block][row block][64][16] and fp32 scales
    [column block][row block][16][128 / group]."""
    n, m = codes.shape
    cb, kb, per = -(-m // 16), -(-n // 128), 128 // group
    packed = np.zeros((cb, kb, 64, 16), np.uint8)
    for j in range(m):
        for i in range(n):
            k = i % 128
            lane, byte = (k % 32) // 8 * 16 + j % 16, k // 32 * 4 + k % 8 // 2
            packed[j // 16, i // 128, lane, byte] |= int(codes[i, j]) << (4 * (k % 2))
    laid = np.zeros((cb, kb, 16, per), np.float32)
    for g in range(scales.shape[0]):
        for j in range(m):
            laid[j // 16, g // per, j % 16, g % per] = scales[g, j]
    return packed, laid
