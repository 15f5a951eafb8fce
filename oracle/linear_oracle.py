"""Independent oracle of the product with an epilogue, of dropout and of the 8-bit format: every operator by its definition, in
64 bits, with numpy on the CPU.  It shares no code with the HIP path."""
import numpy as np

from oracle.block_oracle import activation, activation_slope


def philox4x32(counter, key, rounds=10):
    """The four words of Philox4x32 (Salmon, Moraes, Dror, Shaw 2011) for counters of shape (..., 4) and a key of two words."""
    c = [np.asarray(counter[..., i], dtype=np.uint64) for i in range(4)]      # (products of 32 x 32 bits fit)
    k = [int(key[0]), int(key[1])]
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> half) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> half) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return np.stack(c, -1)


def kept(rows, cols, p, seed, offset=0):
    """Which entries dropout keeps; rows and cols: numbers of them, or index arrays."""
    rows = np.arange(rows) if np.isscalar(rows) else np.asarray(rows)
    cols = np.arange(cols) if np.isscalar(cols) else np.asarray(cols)
    quads, place = np.unique(cols // 4, return_inverse=True)
    offset %= 2 ** 64
    seed %= 2 ** 64
    counter = np.empty((len(rows), len(quads), 4), dtype=np.uint64)
    counter[..., 0], counter[..., 1] = quads[None], rows[:, None]
    counter[..., 2], counter[..., 3] = offset % 2 ** 32, offset // 2 ** 32
    words = philox4x32(counter, (seed % 2 ** 32, seed // 2 ** 32))
    return words[:, place, cols % 4] >= min(round(p * 2 ** 32), 2 ** 32 - 1)


def dropout(x, p, seed, offset=0, residual=0.0):
    return residual + np.where(kept(*x.shape, p, seed, offset), x / (1 - p), 0.0) if p > 0 else residual + x


def linear(X, W, bias=None, residual=0.0, act=None, drop=None):
    """Y, Z; drop: (p, seed, offset)."""
    Z = np.asarray(X, np.float64) @ np.asarray(W, np.float64)
    if bias is not None:
        Z = Z + bias
    V = Z if act is None else activation(act, Z)
    return residual + (V if drop is None else dropout(V, *drop)), Z


def linear_backward(dY, X, W, Z=None, act=None, drop=None):
    """dX, dW, dbias, and the gradient dZ they come from."""
    dZ = np.asarray(dY, np.float64) if drop is None else dropout(np.asarray(dY, np.float64), *drop)
    if act is not None:
        dZ = dZ * activation_slope(act, np.asarray(Z, np.float64))
    if drop is not None:      # (a dropped entry's is zero at a NaN, too)
        dZ = np.where(kept(*dZ.shape, *drop), dZ, 0.0)
    return dZ @ np.asarray(W, np.float64).T, np.asarray(X, np.float64).T @ dZ, dZ.sum(0), dZ


# ---------------------------------------------------------------- 8 bits

def e8m0(top):
    """The smallest power of two, 2^-127 at least, with which magnitudes up to `top` are at most 448."""
    f, k = np.frexp(top)                       # top = f 2^k, 1/2 <= f < 1; 448 = 7/8 2^9
    return np.exp2(np.where(top > 0, np.maximum(np.where(f > 0.875, k - 8, k - 9), -127), -127).astype(np.float64))


def e4m3(v):
    """Values of at most 448 in magnitude, rounded to the nearest code's value, ties to the even one."""
    _, k = np.frexp(np.abs(v))
    step = np.exp2(np.maximum(k - 1, -6) - 3.0)
    return np.rint(v / step) * step


def blocks(n):
    return -(-n // 128) * 128


def pack8(A):
    """Codes' values (rows x whole blocks) and scales of a matrix; groups with a NaN or an infinity are NaN, their scale 1."""
    A = np.asarray(A, np.float64)
    rows, n = A.shape
    full = np.zeros((rows, blocks(n)))
    full[:, :n] = A
    g = full.reshape(rows, -1, 32)
    bad = ~np.isfinite(g).all(2)
    top = np.where(bad, 0.0, np.abs(np.where(np.isfinite(g), g, 0.0)).max(2))
    s = np.where(bad, 1.0, e8m0(top))
    codes = np.where(bad[..., None], np.nan, e4m3(np.where(bad[..., None], 0.0, g) / s[..., None]))
    return codes.reshape(rows, -1), s


def unpack8(codes, scales, n):
    rows = codes.shape[0]
    return (codes.reshape(rows, -1, 32) * scales[..., None]).reshape(rows, -1)[:, :n]
