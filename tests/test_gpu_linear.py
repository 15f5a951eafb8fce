"""GPU parity of the product with an epilogue, its gradients, dropout, the norm with its output in 8 bits and the 8-bit products
against the 64-bit oracle.

Tolerances are bounds, as in test_gpu_block: (2 K + 64) u sum|a||b| for a sum of K products in fp32, 16 u of an elementary
function's value, the unit roundoff of the storage type for a result.  Beside them: gelu with 16-bit results takes an approximation of
Phi(-|z|) that is off by 5e-5 of itself above -3, 1e-3 above -4.5, 4e-3 above -6; the matrix cores' 8-bit sums keep 16 bits beside the
largest of eight products, 2^-13 sum|a||b|; an e4m3 code is half a step off, 2^-4 of the value or 2^-10 of the scale."""
import importlib.util
import os

import numpy as np
import pytest

from oracle import block_oracle as bo
from oracle import linear_oracle as lo
from test_gpu_block import ROUND, TYPES, U32, close, matrix, mp, pools, stored, sum_bound, values  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SLOPE = 1.13               # of both smooth activations, at most
ACTS = [None, "silu", "gelu", "relu"]
SIZES = [(1, 1, 1), (2, 3, 5), (16, 256, 128), (1, 40, 300), (5, 129, 1000), (17, 33, 65), (31, 520, 72), (64, 64, 64), (65, 127, 129),
         (128, 128, 128), (129, 200, 257), (200, 1001, 130), (257, 72, 520), (300, 264, 1032), (520, 512, 640)]


def gelu_short(act, dtype, z):
    """How far the 16-bit form of Phi(-|z|) may be off, relative to it."""
    if act != "gelu" or dtype == "f32":
        return 0.0
    return np.where(z > -3, 5e-5, np.where(z > -4.5, 1e-3, np.where(z > -6, 4e-3, 1.0)))


def guarded(rows, cols, dtype, gap=3):
    """An output in the middle of sevens, and a check that they are still there."""
    pad = torch.full((rows + 2, cols + gap), 7.0, dtype=TYPES[dtype], device="cuda")

    def intact():
        assert (pad[0] == 7).all() and (pad[rows + 1] == 7).all() and (pad[:, cols:] == 7).all(), "written outside"
    return pad[1:rows + 1, :cols], intact


def dropped(mp, rng, p):
    seed, offset = int(rng.integers(0, 2 ** 63)) * 2 + 1, int(rng.integers(0, 2 ** 63))
    return (mp.Dropout(p, seed, offset), (p, seed, offset)) if p else (None, None)


def workspace(mp, nbytes):
    ws = mp.Workspace(nbytes)
    ws.buf.fill_(255)
    return ws


def forward_bounds(x, w, bias, res, act, drop, dtype, K):
    """Y, Z and how far each may be off."""
    Y, Z = lo.linear(x, w, bias, res, act, drop)
    eZ = sum_bound(K + 1, dtype) * (np.abs(x) @ np.abs(w) + (0 if bias is None else np.abs(bias)))
    V = Z if act is None else bo.activation(act, Z)
    eV = eZ if act is None else SLOPE * eZ + 16 * U32 * (np.abs(V) + np.abs(Z)) + gelu_short(act, dtype, Z) * np.abs(V)
    if drop is not None:
        V, eV = lo.dropout(V, *drop), lo.dropout(eV, *drop)
    return Y, Z, eV + 4 * U32 * (np.abs(V) + np.abs(res)) + stored(Y, dtype), eZ + stored(Z, dtype)


def check_forward(mp, rng, tokens, n, m, dtype, act=None, bias=False, residual=False, p=0.0, saved=False, gap=0, in_place=False):
    (X, x), (W, w) = matrix(rng, tokens, n, dtype, gap=gap), matrix(rng, n, m, dtype, n ** -0.5, gap)
    B, b = (t[0] for t in matrix(rng, 1, m, dtype)) if bias else (None, None)
    R, r = matrix(rng, tokens, m, dtype, 2.0, gap) if residual else (None, 0.0)
    drop, plain = dropped(mp, rng, p)
    Y, Z, eY, eZ = forward_bounds(x, w, b, r, act, plain, dtype, n)
    out, intact = guarded(tokens, m, dtype)
    z, z_intact = guarded(tokens, m, dtype, 5) if saved else (None, None)
    if in_place:
        out.copy_(R)
        R = out
    got = mp.linear(X, W, bias=B, residual=R, act=act, dropout=drop, Y=out, z_out=z, workspace=workspace(mp, mp.linear_workspace_bytes(tokens, n, m, TYPES[dtype])))
    torch.cuda.synchronize()
    assert got.data_ptr() == out.data_ptr()
    close(out, Y, eY, "Y")
    intact()
    if saved:
        close(z, Z, eZ, "Z")
        z_intact()
    if p and not residual:
        np.testing.assert_array_equal(values(out)[~lo.kept(tokens, m, *plain)], 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("i", range(len(SIZES)))
def test_linear_forward(mp, i, dtype):  # noqa: F811
    rng = np.random.default_rng(100 + i)
    for k, act in enumerate(ACTS):
        check_forward(mp, rng, *SIZES[i], dtype, act, bias=k % 2 == 0, residual=k < 2, p=(0.0, 0.3, 0.5, 0.1)[(k + i) % 4],
                      saved=(k + i) % 3 == 0, gap=(0, 8, 1, 0)[(k + i) % 4], in_place=k == 1)


def check_backward(mp, rng, tokens, n, m, dtype, act=None, p=0.0, gap=0, need=(True, True, True)):
    (X, x), (W, w) = matrix(rng, tokens, n, dtype, gap=gap), matrix(rng, n, m, dtype, n ** -0.5, gap)
    dY, dy = matrix(rng, tokens, m, dtype, gap=gap)
    Z, z = matrix(rng, tokens, m, dtype, gap=gap) if act else (None, None)
    drop, plain = dropped(mp, rng, p)
    dX, dW, dbias, dZ = lo.linear_backward(dy, x, w, z, act, plain)
    up = np.abs(dy if plain is None else lo.dropout(dy, *plain))
    e_slope = 0 if act in (None, "relu") else 32 * U32 * (1 + np.abs(z)) + (2.5e-5 if act == "gelu" and dtype != "f32" else 0)
    exact = up * e_slope + 4 * U32 * np.abs(dZ)
    e = exact + (stored(dZ, dtype) + ROUND[dtype] * exact if act or p else 0)
    aw, ax = np.abs(w), np.abs(x)
    bx = e @ aw.T + sum_bound(m, dtype) * ((np.abs(dZ) + e) @ aw.T)
    bw = ax.T @ e + sum_bound(tokens, dtype) * (ax.T @ (np.abs(dZ) + e))
    bb = exact.sum(0) + (2 * tokens + 64) * U32 * (np.abs(dZ) + exact).sum(0)
    outs = [guarded(tokens, n, dtype), guarded(n, m, dtype)]
    got = mp.linear_backward(dY, X, W, Z=Z, act=act, dropout=drop, dX=outs[0][0], dW=outs[1][0],
                             workspace=workspace(mp, mp.linear_workspace_bytes(tokens, n, m, TYPES[dtype], True)), need_dx=need[0], need_dw=need[1],
                             need_dbias=need[2])
    torch.cuda.synchronize()
    for k, (want, bound, what) in enumerate(((dX, bx + stored(dX, dtype), "dX"), (dW, bw + stored(dW, dtype), "dW"), (dbias, bb + 1e-37, "dbias"))):
        if need[k]:
            close(got[k], want, bound, what)
        else:
            assert got[k] is None
    for _, intact in outs:
        intact()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("i", range(len(SIZES)))
def test_linear_backward(mp, i, dtype):  # noqa: F811
    rng = np.random.default_rng(200 + i)
    for k, act in enumerate(ACTS):
        check_backward(mp, rng, *SIZES[i], dtype, act, p=(0.0, 0.3)[(k + i) % 2], gap=(0, 8, 1, 0)[(k + i) % 4],
                       need=((True, True, True), (True, False, False), (False, True, True), (False, False, True))[(k + i) % 4])


@pytest.mark.parametrize("tokens,n,m", [(1, 4096, 2048), (40, 2048, 1024), (700, 1536, 1280), (2048, 1024, 1536), (1100, 520, 4104)])
def test_linear_larger(mp, tokens, n, m):  # noqa: F811
    rng = np.random.default_rng(300)
    check_forward(mp, rng, tokens, n, m, "bf16", "gelu", bias=True, residual=True, p=0.1, saved=True)
    check_backward(mp, rng, tokens, n, m, "bf16", "silu", p=0.1)


@pytest.mark.parametrize("act", [None, "silu", "gelu"])
def test_linear_gradients_are_differences(mp, act):  # noqa: F811
    """Of L = sum dY Y along a direction of W, of X and of the bias, from outputs in fp32."""
    rng = np.random.default_rng(301)
    tokens, n, m, h = 37, 50, 44, 2.0 ** -4
    (X, x), (W, w), (B, b) = matrix(rng, tokens, n, "f32"), matrix(rng, n, m, "f32", n ** -0.5), matrix(rng, 1, m, "f32")
    dY, dy = matrix(rng, tokens, m, "f32")
    drop, plain = dropped(mp, rng, 0.25)
    Z = torch.empty_like(dY)
    mp.linear(X, W, bias=B[0], act=act, dropout=drop, z_out=Z)
    grads = mp.linear_backward(dY, X, W, Z=Z, act=act, dropout=drop, need_dbias=True)
    keep = lo.kept(tokens, m, *plain) / 0.75
    for k, (t, v) in enumerate(((X, x), (W, w), (B, b))):
        D, d = matrix(rng, *t.shape, "f32", 0.5 / v.shape[0] ** 0.5)
        loss, noise = [], 0.0
        for sign in (1.0, -1.0):
            moved = [X, W, B]
            moved[k] = t + sign * h * D
            mv = values(moved[k])
            a = [x, w, b]
            a[k] = mv
            _, _, eY, _ = forward_bounds(a[0], a[1], a[2][0], 0.0, act, plain, "f32", n)
            loss.append(float((values(mp.linear(moved[0], moved[1], bias=moved[2][0], act=act, dropout=drop)) * dy).sum()))
            noise += float((np.abs(dy) * eY).sum()) / (2 * h)
        difference = (loss[0] - loss[1]) / (2 * h)
        g = values(grads[k]).reshape(v.shape)
        step = np.abs(h * d @ w if k == 0 else x @ (h * d) if k == 1 else h * d) + 1e-6
        # central differences leave |step|^3 / 6 of the third derivative (at most 2 for both activations); moved arrays are rounded
        bent = 0.0 if act is None else float((np.abs(dy) * keep * step ** 3).sum()) / 3 / h
        rounded = float((np.abs(g) * 2 * U32 * (np.abs(v) + np.abs(d))).sum()) / h
        assert abs(difference - float((g * d).sum())) <= noise + bent + rounded + 1e-5 * float(np.abs(g * d).sum())


def test_linear_non_finite_inputs_stay_in_their_rows(mp):  # noqa: F811
    rng = np.random.default_rng(302)
    for dtype, tokens in (("bf16", 20), ("f16", 200), ("f32", 20), ("f32", 200)):
        (X, x), (W, w) = matrix(rng, tokens, 136, dtype), matrix(rng, 136, 264, dtype)
        R, _ = matrix(rng, tokens, 264, dtype)
        before = mp.linear(X, W, residual=R)
        X[3, 5] = float("nan")
        X[11, 100] = float("inf")
        R[6, 7] = float("-inf")
        after = mp.linear(X, W, residual=R)
        torch.cuda.synchronize()
        rest = [i for i in range(tokens) if i not in (3, 6, 11)]
        assert torch.equal(after[rest], before[rest])
        assert torch.isnan(after[3]).all()
        signs = torch.sign(W[100].float()) * float("inf")
        assert torch.equal(after[11].float(), signs), dtype
        assert after[6, 7] == float("-inf") and torch.equal(after[6, :7], before[6, :7]) and torch.equal(after[6, 8:], before[6, 8:])


def test_dropped_entries_are_zeros_whatever_they_were(mp):  # noqa: F811
    rng = np.random.default_rng(303)
    drop, plain = dropped(mp, rng, 0.5)
    for dtype in TYPES:
        x, _ = matrix(rng, 9, 37, dtype)
        x[2] = float("nan")
        x[4] = float("inf")
        keep = torch.from_numpy(lo.kept(9, 37, *plain)).cuda()
        y = mp.dropout(x, drop)
        assert not y[~keep].any() and torch.isnan(y[2][keep[2]]).all() and torch.isinf(y[4][keep[4]]).all()
        # the same as a product's epilogue
        z = mp.linear(x[:, :1].contiguous(), torch.ones(1, 37, dtype=TYPES[dtype], device="cuda"), dropout=drop)
        assert not z[~keep].any() and torch.isnan(z[2][keep[2]]).all() and torch.isinf(z[4][keep[4]]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens,n", [(1, 1), (1, 5), (3, 7), (4, 64), (33, 100), (100, 1001), (257, 4096), (5, 20000)])
def test_dropout(mp, tokens, n, dtype):  # noqa: F811
    rng = np.random.default_rng(304)
    for p, residual, gap in ((0.1, True, 0), (0.5, False, 1), (0.999, True, 8), (0.0, True, 0), (2.0 ** -40, False, 0)):
        X, x = matrix(rng, tokens, n, dtype, gap=gap)
        R, r = matrix(rng, tokens, n, dtype, gap=gap) if residual else (None, 0.0)
        seed, offset = int(rng.integers(0, 2 ** 63)) * 2 + 1, int(rng.integers(0, 2 ** 63)) * 2
        drop = mp.Dropout(p, seed, offset)
        V = lo.dropout(x, p, seed, offset)
        bound = 4 * U32 * (np.abs(V) + np.abs(r)) + stored(r + V, dtype)
        out, intact = guarded(tokens, n, dtype)
        got = mp.dropout(X, drop, residual=R, y=out)
        torch.cuda.synchronize()
        assert got.data_ptr() == out.data_ptr()
        close(out, r + V, bound, "y")
        intact()
        assert torch.equal(mp.dropout(X, drop, residual=R), out)
        assert torch.equal(mp.dropout_backward(X, drop), mp.dropout(X, drop))
        # in place, over either input
        a = X.clone()
        assert mp.dropout(a, drop, residual=R, y=a) is a and torch.equal(a, out)
        if residual:
            b = R.clone()
            assert torch.equal(mp.dropout(X, drop, residual=b, y=b), out)


def test_dropout_is_the_same_mask_in_a_product_s_epilogue(mp):  # noqa: F811
    """For every way a product is computed: straight tiles of each size, shares of the sum, staged tiles, few fp32 tokens."""
    rng = np.random.default_rng(305)
    for tokens, n, m, dtype in ((300, 264, 1032, "bf16"), (2048, 1024, 1536, "bf16"), (1, 4096, 512, "bf16"), (70, 8192, 136, "f16"), (129, 33, 257, "bf16"),
                                (5, 129, 1000, "f32"), (200, 72, 520, "f32")):
        X, W = matrix(rng, tokens, n, dtype)[0], matrix(rng, n, m, dtype, n ** -0.5)[0]
        drop, plain = dropped(mp, rng, 0.4)
        ones, zero = torch.ones(tokens, m, dtype=TYPES[dtype], device="cuda"), torch.zeros(n, m, dtype=TYPES[dtype], device="cuda")
        bias = torch.ones(m, dtype=TYPES[dtype], device="cuda")
        assert torch.equal(mp.linear(X, zero, bias=bias, dropout=drop), mp.dropout(ones, drop))
        dropped_y, whole = mp.linear(X, W, dropout=drop), mp.linear(X, W)
        keep = torch.from_numpy(lo.kept(tokens, m, *plain)).cuda()
        assert not dropped_y[~keep].any() and (dropped_y[keep] != 0).sum() == (whole[keep] != 0).sum()


def test_dropout_step_on_the_device_moves_a_captured_mask(mp):  # noqa: F811
    rng = np.random.default_rng(306)
    X, x = matrix(rng, 40, 264, "bf16")
    W, _ = matrix(rng, 264, 136, "bf16")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    drop = mp.Dropout(0.5, 99, 2 ** 33, step=step)
    y, h, dx = torch.empty_like(X), torch.empty(40, 136, dtype=X.dtype, device="cuda"), torch.empty_like(X)
    ws = [mp.Workspace(mp.linear_workspace_bytes(40, 264, 136, X.dtype, back)) for back in (False, True)]

    def calls():
        mp.dropout(X, drop, y=y)
        mp.linear(X, W, dropout=drop, Y=h, workspace=ws[0])
        mp.linear_backward(h, X, W, dropout=drop, dX=dx, need_dw=False, workspace=ws[1])
        step.add_(1)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    step.fill_(0)
    with torch.cuda.graph(graph):
        calls()
    for turn in range(4):
        at = int(step.item())
        graph.replay()
        torch.cuda.synchronize()
        fixed = mp.Dropout(0.5, 99, 2 ** 33 + at)
        assert torch.equal(y, mp.dropout(X, fixed))
        assert torch.equal(h, mp.linear(X, W, dropout=fixed))
        assert torch.equal(dx, mp.linear_backward(h, X, W, dropout=fixed, need_dw=False)[0])
        np.testing.assert_array_equal(values(y) != 0, lo.kept(40, 264, 0.5, 99, 2 ** 33 + at) & (x != 0))
        assert int(step.item()) == at + 1


# ---------------------------------------------------------------- 8 bits

def codes_of(q):
    """A Q8's codes as values, scales, and the matrix they stand for."""
    c, s = q.codes.float().cpu().double().numpy(), q.scales.float().cpu().double().numpy()
    return c, s, lo.unpack8(c, s, q.n)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,n", [(1, 1), (3, 31), (2, 32), (5, 33), (16, 128), (7, 129), (40, 1000), (300, 257), (2, 5000)])
def test_q8_pack(mp, rows, n, dtype):  # noqa: F811
    """To the bit: a scale is a comparison of bits, and codes are one rounding of exact quotients."""
    rng = np.random.default_rng(400)
    spread = np.exp2(rng.integers(-9, 6, (rows, 1)))
    A, a = matrix(rng, rows, n, dtype, gap=3)
    A.mul_(torch.from_numpy(spread).to(A.dtype).cuda())
    if n > 40:
        A[0, :40] = 0
    a = values(A)
    want, scales = lo.pack8(a)
    for q in (mp.q8_pack(A), mp.q8_pack(A.t().contiguous(), columns=True)):
        c, s, _ = codes_of(q)
        np.testing.assert_array_equal(s, scales)
        np.testing.assert_array_equal(c, want)
        assert q.rows == rows and q.n == n
    back = lo.unpack8(want, scales, n)
    assert (np.abs(back - a) <= np.maximum(np.abs(a) * 2.0 ** -4, np.repeat(scales, 32, 1)[:, :n] * 2.0 ** -10)).all()


def test_q8_pack_extremes(mp):  # noqa: F811
    tiny, big = 2.0 ** -149, 3.4028234663852886e38
    for top in (0.0, tiny, 2.0 ** -126, 2.0 ** -119, 2.0 ** -118, 1.75 * 2.0 ** -118, 448.0, np.nextafter(np.float32(448), np.float32(999)), 1.75, 1.0, 2.0 ** 120, big):
        a = np.zeros((4, 160), np.float32)
        a[0, 0], a[1, 33], a[2, 159], a[3, :32] = top, -top, top, np.float32(top) * np.linspace(-1, 1, 32, dtype=np.float32)
        want, scales = lo.pack8(a)
        for q in (mp.q8_pack(torch.from_numpy(a).cuda()), mp.q8_pack(torch.from_numpy(a.T.copy()).cuda(), columns=True)):
            c, s, _ = codes_of(q)
            np.testing.assert_array_equal(s, scales)
            np.testing.assert_array_equal(c, want)
    for dtype in TYPES:
        A = torch.ones(3, 100, dtype=TYPES[dtype], device="cuda")
        A[0, 40], A[1, 99], A[2, 0] = float("nan"), float("inf"), float("-inf")
        want, scales = lo.pack8(values(A))
        for q in (mp.q8_pack(A), mp.q8_pack(A.t().contiguous(), columns=True)):
            c, s, _ = codes_of(q)
            np.testing.assert_array_equal(c, want)
            np.testing.assert_array_equal(s, scales)
            assert np.isnan(c).sum() == 32 * 3


NORM8_SIZES = [(1, 1), (3, 31), (2, 64), (5, 65), (9, 128), (4, 300), (17, 1000), (3, 1024), (2, 2047), (6, 4096), (3, 8200), (2, 16384), (2, 17000), (2, 33000)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("i", range(len(NORM8_SIZES)))
def test_block_norm8(mp, i, dtype):  # noqa: F811
    """r is block_norm's to the bit; codes are half a step of the definition's y off, and scales the smallest, both up to what
    fp32 leaves of y (4 n + 200 roundings: two sums of squares, their roots, a dozen products)."""
    tokens, n = NORM8_SIZES[i]
    rng = np.random.default_rng(500 + i)
    for k, (block, token_gate, gap) in enumerate(((True, False, 0), (True, True, 3), (False, False, 1))):
        X, x = matrix(rng, tokens, n, dtype, gap=gap)
        Wp, wp = (t[0] for t in matrix(rng, 1, n, dtype))
        args, plain = {}, {}
        if block:
            B, b = matrix(rng, tokens, n, dtype, gap=gap)
            Wb, wb = (t[0] for t in matrix(rng, 1, n, dtype))
            G, g = matrix(rng, tokens, n, dtype, gap=gap) if token_gate else (t[0] for t in matrix(rng, 1, n, dtype))
            args, plain = dict(b=B, w_post=Wb, gate=G), dict(b=b, w_post=wb, gate=g)
        r, q = mp.block_norm8(X, w_pre=Wp, scale=0.5, **args)
        torch.cuda.synchronize()
        if block:
            assert torch.equal(r, mp.block_norm(X, w_pre=Wp, scale=0.5, **args)[0])
        else:
            assert r is X
        if dtype == "f32":
            # the same numbers as fp32 y, packed
            want = mp.q8_pack(mp.block_norm(X, w_pre=Wp, scale=0.5, **args)[1])
            assert torch.equal(q.codes.view(torch.uint8), want.codes.view(torch.uint8)) and torch.equal(q.scales.view(torch.uint8), want.scales.view(torch.uint8))
        R, y = bo.block_norm(x, w_pre=wp, scale=0.5, **plain)
        c, s, got = codes_of(q)
        off = (4 * n + 200) * U32
        # (r is a sum that may cancel: its error is relative to the parts')
        parts = np.abs(x) + (np.abs(R - x) if block else 0)
        e = off * (np.abs(y) + np.abs(wp) * parts / bo.rms(R, 1e-6))
        group = np.zeros((2,) + c.shape)
        group[0, :, :n], group[1, :, :n] = np.maximum(np.abs(y) - e, 0), np.abs(y) + e
        low, high = (lo.e8m0(v.reshape(tokens, -1, 32).max(2)) for v in group)
        assert ((s >= low) & (s <= high)).all()
        step = np.repeat(s, 32, 1)[:, :n]
        close(torch.from_numpy(got), y, e + np.maximum((np.abs(y) + e) * 2.0 ** -4, step * 2.0 ** -10), "y")
        assert not c[:, n:].any()


def test_block_norm8_non_finite_and_zero_rows(mp):  # noqa: F811
    for dtype in TYPES:
        x = torch.ones(4, 200, dtype=TYPES[dtype], device="cuda")
        x[1, 5], x[2, 7], x[3] = float("nan"), float("inf"), 0.0
        w = torch.ones(200, dtype=TYPES[dtype], device="cuda")
        c, s, got = codes_of(mp.block_norm8(x, w_pre=w)[1])
        assert np.isnan(got[1]).all() and not got[3].any() and np.isfinite(got[0]).all()
        # an infinite entry: rms infinite, itself NaN and the others zeros; its group is NaN
        assert np.isnan(got[2, :32]).all() and not got[2, 32:].any()
        # a row of zeros without eps is 0 / 0
        assert np.isnan(codes_of(mp.block_norm8(x, w_pre=w, eps=0.0)[1])[2][3]).all()
        # past the row: zeros, but in the group that is NaN
        assert not c[[0, 2, 3], 200:].any() and np.isnan(c[1, 200:224]).all() and not c[1, 224:].any()


Q8_SIZES = [(1, 1, 1), (1, 4096, 300), (3, 33, 70), (16, 200, 16), (16, 8192, 48), (17, 128, 65), (40, 300, 129), (64, 1000, 64), (65, 129, 200), (129, 513, 257),
            (300, 2000, 520), (520, 640, 1032), (2, 5000, 2100), (257, 100, 4104), (31, 16500, 24)]


def q8_case(mp, rng, tokens, n, m, gap=0):
    x = mp.q8_pack(matrix(rng, tokens, n, "f32")[0])
    w = mp.q8_pack(matrix(rng, n, m, "f32", n ** -0.5)[0], columns=True)
    if gap:      # rows further apart
        both = []
        for q in (x, w):
            wide, groups = q.codes.shape[1], q.scales.shape[1]
            codes = torch.full((q.rows, wide + 16 * gap), 127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
            scales = torch.full((q.rows, groups + 4 * gap), 255, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
            codes[:, :wide].copy_(q.codes)
            scales[:, :groups].copy_(q.scales)
            both.append(mp.Q8(n, codes[:, :wide], scales[:, :groups]))
        x, w = both
    return x, codes_of(x)[2], w, codes_of(w)[2].T


def q8_bound(x, w, dtype):
    a = np.abs(x) @ np.abs(w)
    return (sum_bound(x.shape[1], "bf16") + (0.0 if dtype == "f32" else 2.0 ** -13)) * a


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("i", range(len(Q8_SIZES)))
def test_q8_products(mp, i, dtype):  # noqa: F811
    tokens, n, m = Q8_SIZES[i]
    rng = np.random.default_rng(600 + i)
    X, x, W, w = q8_case(mp, rng, tokens, n, m, gap=i % 3)
    for k, act in enumerate(ACTS):
        bias, residual = k % 2 == 0, k < 2
        B, b = (t[0] for t in matrix(rng, 1, m, dtype)) if bias else (None, 0.0)
        R, r = matrix(rng, tokens, m, dtype, gap=k) if residual else (None, 0.0)
        Z = x @ w + b
        eZ = q8_bound(x, w, dtype) + 2 * U32 * np.abs(Z)
        V = Z if act is None else bo.activation(act, Z)
        eV = eZ if act is None else SLOPE * eZ + 16 * U32 * (np.abs(V) + np.abs(Z)) + gelu_short(act, dtype, Z) * np.abs(V)
        out, intact = guarded(tokens, m, dtype)
        got = mp.q8_linear(X, W, bias=B, residual=R, act=act, y=out, workspace=workspace(mp, mp.q8_workspace_bytes(tokens, n, m)))
        torch.cuda.synchronize()
        assert got is out
        close(out, r + V, eV + 4 * U32 * (np.abs(V) + np.abs(r)) + stored(r + V, dtype), "y")
        intact()
        if residual:
            c = R.clone()
            assert torch.equal(mp.q8_linear(X, W, bias=B, residual=c, act=act, y=c), out)
    U = mp.Q8(n, torch.flip(W.codes.view(torch.uint8), (0,)).view(torch.float8_e4m3fn), torch.flip(W.scales.view(torch.uint8), (0,)).view(torch.float8_e8m0fnu))
    W = mp.Q8(n, W.codes.contiguous(), W.scales.contiguous())
    u = w[:, ::-1]
    for act in ACTS[1:]:
        g, up = x @ w, x @ u
        e, eu = q8_bound(x, w, dtype), q8_bound(x, u, dtype)
        a = bo.activation(act, g)
        out, intact = guarded(tokens, m, dtype)
        mp.q8_gated(X, W, U, act=act, h=out, workspace=workspace(mp, mp.q8_workspace_bytes(tokens, n, m, True)))
        torch.cuda.synchronize()
        ea = SLOPE * e + 16 * U32 * (np.abs(a) + np.abs(g)) + gelu_short(act, dtype, g) * np.abs(a)
        close(out, a * up, ea * (np.abs(up) + eu) + np.abs(a) * eu + 2 * U32 * np.abs(a * up) + stored(a * up, dtype), "h")
        intact()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens,n,m", [(1, 640, 40), (16, 128, 64), (40, 256, 136), (130, 300, 257), (300, 1024, 520), (600, 384, 2056), (1500, 128, 4100)])
def test_q8_products_of_whole_numbers_are_exact(mp, tokens, n, m, dtype):  # noqa: F811
    """Products of up to 16, and sums below the type's whole numbers, with scales 2^-1, 1 and 2 that differ from group to group: every one is
    exact however the matrix cores add."""
    rng = np.random.default_rng(700)
    size = {"bf16": 2 ** 8, "f16": 2 ** 11, "f32": 2 ** 24}[dtype]
    density = min(1.0, size / 4 / (4 * 16) / n * 8)
    def sparse(rows):
        v = rng.integers(-4, 5, (rows, -(-n // 32), 32)) * (rng.random((rows, -(-n // 32), 32)) < density ** 0.5)
        return v.reshape(rows, -1)[:, :n].astype(np.float32)
    x, w = sparse(tokens), sparse(m)
    X, W = mp.q8_pack(torch.from_numpy(x).cuda()), mp.q8_pack(torch.from_numpy(w).cuda())
    np.testing.assert_array_equal(codes_of(X)[2], x)
    want = x.astype(np.float64) @ w.T.astype(np.float64)
    assert np.abs(want).max() <= size
    np.testing.assert_array_equal(values(mp.q8_linear(X, W, dtype=TYPES[dtype])), want)
    h = mp.q8_gated(X, W, W, act="relu", dtype=torch.float32)
    np.testing.assert_array_equal(values(h), np.maximum(want, 0) * want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens", [1, 20, 300])
def test_q8_products_keep_a_nan_in_its_row_or_column(mp, tokens, dtype):  # noqa: F811
    rng = np.random.default_rng(701)
    A, B = matrix(rng, tokens, 300, "f32")[0], matrix(rng, 300, 200, "f32")[0]
    before = mp.q8_linear(mp.q8_pack(A), mp.q8_pack(B, columns=True), dtype=TYPES[dtype])
    B[7, 33] = float("inf")
    if tokens > 1:
        A[tokens - 2, 299] = float("nan")
    after = mp.q8_linear(mp.q8_pack(A), mp.q8_pack(B, columns=True), dtype=TYPES[dtype])
    bad = torch.zeros_like(after, dtype=torch.bool)
    bad[:, 33] = True
    if tokens > 1:
        bad[tokens - 2] = True
    assert torch.isnan(after[bad]).all() and torch.equal(after[~bad], before[~bad])


def test_q8_products_larger(mp):  # noqa: F811
    """Whole turns of large tiles, against fp64 on the device."""
    rng = np.random.default_rng(702)
    for tokens, n, m, dtype in ((2100, 4096, 4200, torch.bfloat16), (4096, 1024, 4096, torch.float16), (600, 2048, 3000, torch.float32)):
        x, w = mp.q8_pack(torch.randn(tokens, n, device="cuda")), mp.q8_pack(torch.randn(n, m, device="cuda") * n ** -0.5, columns=True)
        wide = lambda q: (q.codes.double().unflatten(1, (-1, 32)) * q.scales.double()[:, :, None]).flatten(1)  # noqa: E731
        a, b = wide(x), wide(w)
        want, size = a @ b.t(), a.abs() @ b.abs().t()
        u = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}[dtype]
        c = (2 * n + 64) * U32 + (0 if dtype == torch.float32 else 2.0 ** -13)
        got = mp.q8_linear(x, w, dtype=dtype).double()
        assert ((got - want).abs() <= c * size + 1.001 * u * want.abs() + 2.0 ** -24).all()
        h, e = mp.q8_gated(x, w, w, act="silu", dtype=dtype).double(), c * size
        s = want * torch.sigmoid(want)
        assert ((h - s * want).abs() <= (SLOPE * e + 32 * U32 * (1 + s.abs())) * (want.abs() + e) + s.abs() * e + 1.001 * u * (s * want).abs() + 2.0 ** -24).all()


# ---------------------------------------------------------------- as they are used

def test_the_block_in_eight_bits(mp):  # noqa: F811
    """norm -> gated products -> packing -> down product into the residual stream, every step from what the one before left."""
    rng = np.random.default_rng(800)
    for tokens, n, m, dtype in ((1, 520, 1100, "bf16"), (40, 264, 600, "f16"), (300, 300, 700, "f32")):
        (X, x), (B, b) = matrix(rng, tokens, n, dtype), matrix(rng, tokens, n, dtype)
        (Wp, wp), (Wq, wq), (G, g) = ((t[0][0], t[1][0]) for t in (matrix(rng, 1, n, dtype) for _ in range(3)))
        weights = [matrix(rng, n, m, dtype, n ** -0.5)[0], matrix(rng, n, m, dtype, n ** -0.5)[0], matrix(rng, m, n, dtype, m ** -0.5)[0]]
        mask = torch.from_numpy((rng.random(m) < 0.6).astype(np.uint8)).cuda()
        for w in weights[:2]:
            w.mul_(mask.to(w.dtype))
        Wg, Wu, Wd = (mp.q8_pack(w, columns=True) for w in weights)
        r, z = mp.block_norm8(X, B, Wp, G, Wq, scale=0.5)
        h = mp.q8_gated(z, Wg, Wu, dtype=TYPES[dtype])
        h8 = mp.q8_pack(h)
        y = mp.q8_linear(h8, Wd, residual=r)
        torch.cuda.synchronize()
        zv, gv, uv, dv, hv = (codes_of(q)[2] for q in (z, Wg, Wu, Wd, h8))
        e, eu = q8_bound(zv, gv.T, dtype), q8_bound(zv, uv.T, dtype)
        p, q = zv @ gv.T, zv @ uv.T
        a = bo.activation("silu", p)
        close(h, a * q, (SLOPE * e + 32 * U32 * (1 + np.abs(p))) * (np.abs(q) + eu) + np.abs(a) * eu + stored(a * q, dtype), "h")
        assert not h[:, mask == 0].any()
        want = values(r) + hv @ dv.T
        close(y, want, q8_bound(hv, dv.T, dtype) + 4 * U32 * np.abs(want) + stored(want, dtype), "y")


def test_the_block_in_training(mp):  # noqa: F811
    """Gradients through norm, gated products and the down product with dropout into the residual stream, against differences of the loss
    in 64 bits (fp32 storage)."""
    rng = np.random.default_rng(801)
    tokens, n, m, act = 23, 24, 40, "silu"
    (X, x), (Wn, wn), (Wg, wg), (Wu, wu), (Wd, wd), (dY, dy) = (matrix(rng, *s, "f32", k) for s, k in (
        ((tokens, n), 1.0), ((1, n), 1.0), ((n, m), n ** -0.5), ((n, m), n ** -0.5), ((m, n), m ** -0.5), ((tokens, n), 1.0)))
    drop, plain = dropped(mp, rng, 0.2)
    _, z = mp.block_norm(X, w_pre=Wn[0])
    G, U = torch.empty(2, tokens, m, device="cuda")
    h = mp.gated_ff(z, Wg, Wu, act=act, g_out=G, u_out=U)
    y = mp.linear(h, Wd, residual=X, dropout=drop)
    dh, dWd, _ = mp.linear_backward(dY, h, Wd, dropout=drop)
    dz, dWg, dWu = mp.gated_ff_backward(dh, z, Wg, Wu, act=act, G=G, U=U)
    dx, _, _, _, dWn = mp.block_norm_backward(dY, dz, X, w_pre=Wn[0])
    torch.cuda.synchronize()

    def loss(x, wn, wg, wu, wd):
        h = bo.gated_ff(bo.block_norm(x, w_pre=wn[0])[1], wg, wu, act)[0]
        return float((lo.linear(h, wd, residual=x, drop=plain)[0] * dy).sum())
    at = [x, wn, wg, wu, wd]
    assert abs(loss(*at) - float((values(y) * dy).sum())) < 1e-4 * float(np.abs(values(y) * dy).sum())
    for k, got in enumerate((dx, dWn, dWg, dWu, dWd)):
        d = rng.standard_normal(at[k].shape) / np.sqrt(at[k].size)
        h = 1e-5
        difference = (loss(*(at[:k] + [at[k] + h * d] + at[k + 1:])) - loss(*(at[:k] + [at[k] - h * d] + at[k + 1:]))) / (2 * h)
        g = values(got).reshape(at[k].shape)
        # sums of 23 to 40 products in fp32, four products deep: 4 (2 40 + 64) u, of each part of the scalar product
        assert abs(difference - float((g * d).sum())) <= 4 * 144 * U32 * 8 * float(np.linalg.norm(g) * np.linalg.norm(d)) + 1e-6


def test_calls_can_be_captured_and_replayed(mp):  # noqa: F811
    rng = np.random.default_rng(802)
    for tokens, n, m, dtype in ((1, 2000, 520, "bf16"), (300, 700, 1000, "bf16"), (20, 300, 200, "f32"), (2100, 1032, 4168, "f16"), (70, 8192, 136, "bf16")):
        X, W = matrix(rng, tokens, n, dtype)[0], matrix(rng, n, m, dtype, n ** -0.5)[0]
        b, w, R = matrix(rng, 1, m, dtype)[0][0], matrix(rng, 1, n, dtype)[0][0], matrix(rng, tokens, m, dtype)[0]
        drop, _ = dropped(mp, rng, 0.3)
        W8 = mp.q8_pack(W, columns=True)
        x8 = mp.q8_pack(X)
        Y, Z, y8, h8, dX, dW, xd = (torch.empty_like(t) for t in (R, R, R, R, X, W, X))
        ws = [mp.Workspace(k) for k in (mp.linear_workspace_bytes(tokens, n, m, X.dtype), mp.linear_workspace_bytes(tokens, n, m, X.dtype, True),
                                        mp.q8_workspace_bytes(tokens, n, m), mp.q8_workspace_bytes(tokens, n, m, True))]
        held = {}

        def calls():
            mp.linear(X, W, bias=b, residual=R, act="gelu", dropout=drop, Y=Y, z_out=Z, workspace=ws[0])
            held["dbias"] = mp.linear_backward(Y, X, W, Z=Z, act="gelu", dropout=drop, dX=dX, dW=dW, need_dbias=True, workspace=ws[1])[2]
            mp.dropout(X, drop, y=xd)
            mp.block_norm8(X, w_pre=w, y=x8)
            mp.q8_linear(x8, W8, bias=b, residual=R, y=y8, workspace=ws[2])
            mp.q8_gated(x8, W8, W8, h=h8, workspace=ws[3])
            mp.q8_pack(X, packed=x8)

        calls()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls()
        captured = held["dbias"]
        outs = (Y, Z, dX, dW, xd, y8, h8, x8.codes.view(torch.uint8), x8.scales.view(torch.uint8))
        for turn in range(3):
            X.copy_(matrix(rng, tokens, n, dtype)[0])
            calls()
            want = [t.clone() for t in outs] + [held["dbias"].clone()]
            for t in outs + (captured,):
                t.fill_(3)
            graph.replay()
            torch.cuda.synchronize()
            for k, (p, q) in enumerate(zip(want, outs + (captured,))):
                assert torch.equal(p, q), k


def test_calls_on_two_streams_at_once(mp):  # noqa: F811
    rng = np.random.default_rng(803)
    X, W = matrix(rng, 200, 1000, "bf16")[0], matrix(rng, 1000, 600, "bf16", 0.03)[0]
    drop, _ = dropped(mp, rng, 0.3)
    W8, x8 = mp.q8_pack(W, columns=True), mp.q8_pack(X)
    calls = [lambda **k: mp.linear(X, W, act="silu", dropout=drop, **k), lambda **k: mp.linear_backward(X[:, :600], X, W, need_dbias=True, dropout=drop, **k)[1],
             lambda **k: mp.q8_linear(x8, W8, **k), lambda **k: mp.q8_gated(x8, W8, W8, **k), lambda **k: mp.dropout(X, drop, **k)]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[c(stream=s) for c in calls for s in streams] for _ in range(4)]
    torch.cuda.synchronize()
    for round_ in got:
        for k, g in enumerate(round_):
            assert torch.equal(g, want[k // 2])


def test_calls_given_a_stream_allocate_on_it(mp, monkeypatch):  # noqa: F811
    side = torch.cuda.Stream()
    scratch = []
    init = mp.Workspace.__init__

    def noted(self, *args, **kw):
        init(self, *args, **kw)
        scratch.append(self.buf)

    monkeypatch.setattr(mp.Workspace, "__init__", noted)
    rng = np.random.default_rng(804)
    X, W = matrix(rng, 20, 72, "bf16")[0], matrix(rng, 72, 136, "bf16")[0]
    dY, w = matrix(rng, 20, 136, "bf16")[0], matrix(rng, 1, 72, "bf16")[0][0]
    torch.cuda.synchronize()
    kw = dict(stream=side)
    drop = mp.Dropout(0.1, 3)
    x8, W8 = mp.q8_pack(X, **kw), mp.q8_pack(W, columns=True, **kw)
    r, z8 = mp.block_norm8(X, X, w, w, w, **kw)
    outs = [x8.codes, x8.scales, W8.codes, W8.scales, r, z8.codes, z8.scales, mp.linear(X, W, **kw), *mp.linear_backward(dY, X, W, need_dbias=True, **kw),
            mp.dropout(X, drop, **kw), mp.dropout_backward(X, drop, **kw), mp.q8_linear(x8, W8, **kw), mp.q8_gated(x8, W8, W8, **kw)]
    assert len(scratch) == 4
    assert set(pools(outs + scratch)) == {side.cuda_stream}


def test_calls_without_tokens(mp):  # noqa: F811
    for dtype in TYPES.values():
        X, W, b = torch.empty(0, 40, dtype=dtype, device="cuda"), torch.ones(40, 30, dtype=dtype, device="cuda"), torch.ones(30, dtype=dtype, device="cuda")
        drop = mp.Dropout(0.1, 3)
        assert mp.linear(X, W, bias=b, dropout=drop).shape == (0, 30)
        dX, dW, dbias = mp.linear_backward(torch.empty(0, 30, dtype=dtype, device="cuda"), X, W, dropout=drop, need_dbias=True)
        assert dX.shape == (0, 40) and not dW.any() and not dbias.any()
        assert mp.dropout(X, drop).shape == (0, 40)
        r, z = mp.block_norm8(X, w_pre=torch.ones(40, dtype=dtype, device="cuda"))
        W8 = mp.q8_pack(W, columns=True)
        assert z.rows == 0 and mp.q8_linear(z, W8, dtype=dtype).shape == (0, 30) and mp.q8_gated(z, W8, W8, dtype=dtype).shape == (0, 30)
        assert mp.q8_pack(X).rows == 0


def test_rows_further_apart_than_32_bits_reach(mp):  # noqa: F811
    """Rows four million entries apart, the last ones past 2^32 entries from the first."""
    rng = np.random.default_rng(805)
    tokens, n, m, far = 1100, 72, 40, 1 << 22
    whole = torch.empty(tokens * far, dtype=torch.bfloat16, device="cuda")
    X = whole.view(tokens, far)[:, :n]
    near = matrix(rng, tokens, n, "bf16")[0]
    X.copy_(near)
    W, w = matrix(rng, n, m, "bf16", n ** -0.5)[0], matrix(rng, 1, n, "bf16")[0][0]
    drop = mp.Dropout(0.3, 5)
    Y = whole.view(tokens, far)[:, 128:128 + m]
    assert torch.equal(mp.linear(X, W, act="gelu", dropout=drop, Y=Y), mp.linear(near, W, act="gelu", dropout=drop))
    dY = Y.contiguous()
    for p, q in zip(mp.linear_backward(Y, X, W, dropout=drop, need_dbias=True), mp.linear_backward(dY, near, W, dropout=drop, need_dbias=True)):
        assert torch.equal(p, q)
    D = whole.view(tokens, far)[:, 256:256 + n]
    assert torch.equal(mp.dropout(X, drop, residual=X, y=D), mp.dropout(near, drop, residual=near))
    (_, p), (_, q) = mp.block_norm8(X, w_pre=w), mp.block_norm8(near, w_pre=w)
    assert torch.equal(p.codes.view(torch.uint8), q.codes.view(torch.uint8)) and torch.equal(p.scales.view(torch.uint8), q.scales.view(torch.uint8))
    p = mp.q8_pack(X)
    W8 = mp.q8_pack(W, columns=True)
    far8 = whole.view(torch.uint8)[:tokens * far].view(tokens, far).view(torch.float8_e4m3fn)[:, 1024:1152]
    far8.view(torch.uint8).copy_(p.codes.view(torch.uint8))
    assert torch.equal(mp.q8_linear(mp.Q8(n, far8, p.scales), W8, residual=Y), mp.q8_linear(p, W8, residual=dY))


def test_refusals_of_the_binding(mp):  # noqa: F811
    X, W = torch.ones(4, 40, device="cuda"), torch.ones(40, 30, device="cuda")
    drop, x8 = mp.Dropout(0.1, 3), mp.q8_pack(X)
    for bad in (lambda: mp.linear(X, W.half()), lambda: mp.linear(X, W[:39]), lambda: mp.linear(X, W, bias=torch.ones(29, device="cuda")),
                lambda: mp.linear(X, W, residual=X), lambda: mp.linear(X.t(), W), lambda: mp.linear(X, W.cpu()), lambda: mp.linear_backward(X[:, :30], X, W, act="silu"),
                lambda: mp.dropout(X, drop, residual=W), lambda: mp.Dropout(0.1, 3, step=torch.zeros(1, device="cuda")), lambda: mp.block_norm8(X),
                lambda: mp.Q8(41, x8.codes[:, :64], x8.scales), lambda: mp.Q8(40, x8.codes.float(), x8.scales), lambda: mp.q8_linear(x8, mp.q8_pack(W)),
                lambda: mp.q8_linear(x8, mp.q8_pack(W, columns=True), y=torch.ones(4, 30, device="cuda"), dtype=torch.float16),
                lambda: mp.q8_gated(x8, mp.q8_pack(W, columns=True), mp.q8_pack(W[:, :29], columns=True)), lambda: mp.q8_pack(X, packed=mp.q8_pack(W))):
        with pytest.raises(AssertionError):
            bad()
    for bad in (lambda: mp.dropout(X, mp.Dropout(1.0, 3)), lambda: mp.linear(X, W, dropout=mp.Dropout(-0.5, 3)),
                lambda: mp.linear(X, W, workspace=type("W", (), {"buf": X, "nbytes": 8})())):
        with pytest.raises(mp.MlprojError):
            bad()


def test_the_example_trains_with_dropout_and_answers_in_eight_bits(mp):  # noqa: F811
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "pruned_block.py")
    spec = importlib.util.spec_from_file_location("pruned_block_8", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    out = example.main(steps=8, dropout=0.1)
    assert np.isfinite([out["first_loss"], out["last_loss"]]).all()
    # each operand's entry is at most 2^-4 off: three products of two operands, the norms between them; errors of random sign add far below
    assert out["eight_bit_error"] < 6 * 2.0 ** -4
    # gradients of the example's step against the oracle's, at the example's rounding of every stage
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    block = example.PrunedBlock(64, 96, gen)
    x = torch.randn(40, 64, generator=gen, device="cuda").to(torch.bfloat16)
    drop = mp.Dropout(0.25, 17, 4)
    y, saved = block.forward(x, drop)
    h, b, db = saved[2], saved[3], torch.randn(40, 64, generator=gen, device="cuda").to(torch.bfloat16)
    _, dWd, _ = mp.linear_backward(db, h, block.w["Wd"], dropout=drop)
    want = lo.linear_backward(values(db), values(h), values(block.w["Wd"]), drop=(0.25, 17, 4))
    e = stored(want[3], "bf16")
    close(dWd, want[1], np.abs(values(h)).T @ e + sum_bound(40, "bf16") * (np.abs(values(h)).T @ (np.abs(want[3]) + e)) + stored(want[1], "bf16"), "dWd")
    B = lo.linear(values(h), values(block.w["Wd"]), drop=(0.25, 17, 4))[0]
    close(b, B, sum_bound(96, "bf16") * (np.abs(values(h)) @ np.abs(values(block.w["Wd"]))) / 0.75 + 4 * U32 * np.abs(B) + stored(B, "bf16"), "b")


def test_linear_whole_turns_of_large_tiles_and_the_rest(mp):  # noqa: F811
    """306 tiles of 256 x 256: one turn of the compute units, and 50 that go out in smaller ones; against fp64 on the device."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    tokens, n, m = 4400, 1024, 4160
    X, W = (torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16) for s in ((tokens, n), (n, m)))
    W = (W.float() * n ** -0.5).to(torch.bfloat16)
    R, b = (torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16) for s in ((tokens, m), (m,)))
    drop = mp.Dropout(0.2, 77, 3)
    x, w, r = X.double(), W.double(), R.double()
    z = x @ w + b.double()
    v = z * torch.sigmoid(z)
    eZ = (2 * n + 66) * U32 * (x.abs() @ w.abs() + b.double().abs())
    keep = mp.dropout(torch.ones(tokens, m, device="cuda"), drop) != 0      # (itself against the oracle elsewhere)
    v, e = torch.where(keep, v / 0.8, 0.0), torch.where(keep, (SLOPE * eZ + 16 * U32 * (v.abs() + z.abs())) / 0.8, 0.0)
    want = r + v
    for out in (None, R.clone()):
        Z = torch.empty_like(R)
        y = mp.linear(X, W, bias=b, residual=R if out is None else out, act="silu", dropout=drop, Y=out, z_out=Z)
        assert ((y.double() - want).abs() <= e + 4 * U32 * (v.abs() + r.abs()) + 2.0 ** -8 * 1.001 * want.abs()).all()
        assert ((Z.double() - z).abs() <= eZ + 2.0 ** -8 * 1.001 * z.abs()).all()
    dY = torch.randn(tokens, m, generator=gen, device="cuda").to(torch.bfloat16)
    dX, dW, dbias = mp.linear_backward(dY, X, W, need_dbias=True)
    d = dY.double()
    for got, a, c in ((dX, d, w.t()), (dW, x.t(), d)):
        exact, size = a @ c, a.abs() @ c.abs()
        assert ((got.double() - exact).abs() <= (2 * a.shape[1] + 64) * U32 * size + 2.0 ** -8 * 1.001 * exact.abs()).all()
    assert ((dbias.double() - d.sum(0)).abs() <= (2 * tokens + 64) * U32 * d.abs().sum(0)).all()


def test_q8_object_is_fixed(mp):  # noqa: F811
    """The library reads the memory that it was made of."""
    A = torch.ones(3, 200, device="cuda")
    packed = mp.q8_pack(A)
    for q in (packed, mp.Q8(200, packed.codes.clone(), packed.scales.clone())):
        for name in ("rows", "n", "codes", "scales"):
            with pytest.raises(AttributeError):
                setattr(q, name, getattr(packed, name))
        assert torch.equal(mp.q8_linear(q, packed, dtype=torch.float32), torch.full((3, 3), 200.0, device="cuda"))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens,n,m", [(300, 40, 1), (1, 300, 40), (1, 1, 1), (7, 33, 5), (65, 127, 129), (300, 264, 1032), (40, 2048, 1024), (520, 512, 640)])
def test_gradients_through_dropout_alone_are_rounded_once(mp, tokens, n, m, dtype):  # noqa: F811
    """dY's entries and zeros are exact in every type, dY / (1 - p) is not: dX and dW are sums in fp32, their factor and one rounding."""
    rng = np.random.default_rng(310)
    for p, gap in ((0.3, 0), (0.1, 1), (0.9, 8)):
        (X, x), (W, w), (dY, dy) = matrix(rng, tokens, n, dtype, gap=gap), matrix(rng, n, m, dtype, n ** -0.5, gap), matrix(rng, tokens, m, dtype, gap=gap)
        drop, plain = dropped(mp, rng, p)
        dX, dW, dbias, dZ = lo.linear_backward(dy, x, w, drop=plain)
        got = mp.linear_backward(dY, X, W, dropout=drop, need_dbias=True)
        for g, want, a, b, K, what in ((got[0], dX, dZ, w.T, m, "dX"), (got[1], dW, x.T, dZ, tokens, "dW")):
            close(g, want, sum_bound(K, dtype) * (np.abs(a) @ np.abs(b)) + 4 * U32 * np.abs(want) + stored(want, dtype), what)
        close(got[2], dbias, (2 * tokens + 64) * U32 * np.abs(dZ).sum(0) + 1e-37, "dbias")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("act", ACTS[1:])
def test_gradients_at_dropped_entries_are_zeros_whatever_z_is(mp, act, dtype):  # noqa: F811
    """A result that was dropped is zero whatever its pre-activation was, so nothing of that reaches a gradient; of one that was kept it does."""
    rng = np.random.default_rng(311)
    tokens, n, m = 33, 40, 52
    (X, _), (W, _), (dY, _), (Z, _) = (matrix(rng, *s, dtype) for s in ((tokens, n), (n, m), (tokens, m), (tokens, m)))
    drop, plain = dropped(mp, rng, 0.5)
    keep = torch.from_numpy(lo.kept(tokens, m, *plain)).cuda()
    want = mp.linear_backward(dY, X, W, Z=Z, act=act, dropout=drop, need_dbias=True)
    for bad in ("nan", "inf", "-inf"):
        z = Z.clone()
        z[~keep] = float(bad)
        for p, q in zip(mp.linear_backward(dY, X, W, Z=z, act=act, dropout=drop, need_dbias=True), want):
            assert torch.equal(p, q), bad
    row, col = (int(i) for i in torch.nonzero(keep)[100])
    z = Z.clone()
    z[row, col] = float("nan")
    dX, dW, dbias = mp.linear_backward(dY, X, W, Z=z, act=act, dropout=drop, need_dbias=True)
    assert torch.isnan(dX[row]).all() and torch.isnan(dW[:, col]).all() and torch.isnan(dbias[col])
    assert torch.isnan(dX).sum() == n and torch.isnan(dW).sum() == n and torch.isnan(dbias).sum() == 1


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("act", ACTS[1:])
def test_slopes_at_infinite_pre_activations_are_their_limits(mp, act, dtype):  # noqa: F811
    """0 and 1, as they are in fp32 from 200 on: the same gradients to the bit."""
    rng = np.random.default_rng(312)
    tokens, n, m = 40, 72, 56
    (X, _), (W, _), (dY, _), (Z, _) = (matrix(rng, *s, dtype) for s in ((tokens, n), (n, m), (tokens, m), (tokens, m)))
    far = {"+": torch.from_numpy(rng.random((tokens, m)) < 0.1).cuda(), "-": torch.from_numpy(rng.random((tokens, m)) < 0.1).cuda()}
    grads = []
    for size in (200.0, float("inf")):
        z = Z.clone()
        for sign, at in far.items():
            z[at] = float(sign + str(size))
        grads.append(mp.linear_backward(dY, X, W, Z=z, act=act, need_dbias=True))
    for p, q in zip(*grads):
        assert torch.isfinite(p).all() and torch.equal(p, q)


@pytest.mark.parametrize("act", ACTS[1:])
def test_pre_activations_past_fp16_have_their_gradients(mp, act):  # noqa: F811
    """A pre-activation of -2^17 is an infinity in fp16, its result zero (relu's and the others' limit) and so is its gradient."""
    X = torch.zeros(3, 8, dtype=torch.float16, device="cuda")
    X[0, 0], X[1, 0], X[2, 1] = -2.0 ** 10, 2.0 ** -10, 1.0
    W = torch.full((8, 16), 2.0 ** 7, dtype=torch.float16, device="cuda")
    Z = torch.empty(3, 16, dtype=torch.float16, device="cuda")
    y = mp.linear(X, W, act=act, z_out=Z)
    assert torch.isinf(Z[0]).all() and torch.isfinite(Z[1:]).all() and not y[0].any()
    dX, dW, dbias = mp.linear_backward(torch.ones_like(y), X, W, Z=Z, act=act, need_dbias=True)
    assert not dX[0].any() and torch.isfinite(dX).all() and torch.isfinite(dW).all() and torch.isfinite(dbias).all()
    # a gated block's saved gate
    U = torch.ones_like(Z)
    dH = torch.ones_like(y)
    got = mp.gated_ff_backward(dH, X, W, W, act=act, G=Z, U=U)
    want = mp.gated_ff_backward(dH, X, W, W, act=act, G=Z.clamp_min(-200), U=U)
    for p, q in zip(got, want):
        # (dX of the last row is 16 (1 + 2^7) 2^7 = 264192, an infinity in fp16)
        assert torch.isfinite(p[:2]).all() and not torch.isnan(p).any() and torch.equal(p, q)


# Pairs in 32 columns per workgroup on both sides of that rule, with a remainder of columns; 64 blocks a round from n = 8065 on, with rounds
# that are not whole, and a second one
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens,n,m", [(5, 300, 4099), (16, 1000, 4128), (4, 520, 4100), (1, 300, 12290), (5, 300, 12301), (16, 1000, 12320),
                                        (8, 4200, 4111), (7, 4200, 4111), (1, 8200, 40), (9, 12345, 33), (16, 16500, 24), (3, 8064, 20)])
def test_q8_products_of_few_tokens_take_every_form(mp, tokens, n, m, dtype):  # noqa: F811
    rng = np.random.default_rng(703)
    X, x, W, w = q8_case(mp, rng, tokens, n, m)
    U, u = q8_case(mp, rng, 1, n, m)[2:]
    (B, b), (R, r) = (matrix(rng, k, m, dtype) for k in (1, tokens))
    Z, e = x @ w + b, q8_bound(x, w, dtype)
    eZ = e + 2 * U32 * np.abs(Z)
    V = bo.activation("gelu", Z)
    eV = SLOPE * eZ + 16 * U32 * (np.abs(V) + np.abs(Z)) + gelu_short("gelu", dtype, Z) * np.abs(V)
    out, intact = guarded(tokens, m, dtype)
    mp.q8_linear(X, W, bias=B[0], residual=R, act="gelu", y=out, workspace=workspace(mp, mp.q8_workspace_bytes(tokens, n, m)))
    torch.cuda.synchronize()
    close(out, r + V, eV + 4 * U32 * (np.abs(V) + np.abs(r)) + stored(r + V, dtype), "y")
    intact()
    g, up, eu = x @ w, x @ u, q8_bound(x, u, dtype)
    a = bo.activation("silu", g)
    ea = SLOPE * e + 16 * U32 * (np.abs(a) + np.abs(g))
    out, intact = guarded(tokens, m, dtype)
    mp.q8_gated(X, W, U, act="silu", h=out, workspace=workspace(mp, mp.q8_workspace_bytes(tokens, n, m, True)))
    torch.cuda.synchronize()
    close(out, a * up, ea * (np.abs(up) + eu) + np.abs(a) * eu + 2 * U32 * np.abs(a * up) + stored(a * up, dtype), "h")
    intact()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens,n,m", [(1, 640, 40), (16, 1200, 64), (7, 9000, 24), (40, 256, 136), (130, 300, 257), (300, 1024, 520), (600, 384, 2056), (1500, 160, 4100)])
def test_q8_products_find_every_group_s_scale(mp, tokens, n, m, dtype):  # noqa: F811
    """Whole numbers whose groups of 32 along n are multiplied by 2^s in x and by 2^-s in w, with another s in every group, and whose rows by powers of
    two of their own: products are exact however the matrix cores add, and another group's or row's scale would show."""
    rng = np.random.default_rng(704)
    size = {"bf16": 2 ** 8, "f16": 2 ** 11, "f32": 2 ** 24}[dtype]
    density = min(1.0, size / 4 / (4 * 16) / n * 8)
    groups = -(-n // 32)
    s = rng.permutation(groups) % 61 - 30
    assert len(set(s)) == min(groups, 61)

    def whole(rows, sign):
        v = rng.integers(-4, 5, (rows, groups, 32)) * (rng.random((rows, groups, 32)) < density ** 0.5)
        v = v.reshape(rows, -1)[:, :n].astype(np.float64)
        of_row = -rng.integers(0, 4, (rows, 1))
        q = mp.q8_pack(torch.from_numpy(v * 2.0 ** of_row * 2.0 ** (sign * np.repeat(s, 32)[:n])).float().cuda())
        return v, of_row, q
    (x, tx, X), (w, tw, W) = whole(tokens, 1), whole(m, -1)
    sums = x @ w.T
    assert np.abs(sums).max() <= size
    want = sums * 2.0 ** (tx + tw.T)
    np.testing.assert_array_equal(values(mp.q8_linear(X, W, dtype=TYPES[dtype])), want)
    h = (np.maximum(want, 0) * want).astype(np.float32)
    np.testing.assert_array_equal(mp.q8_gated(X, W, W, act="relu", dtype=torch.float32).cpu().numpy(), h)


@pytest.mark.parametrize("tokens", [1, 20])
def test_q8_products_at_the_ends_of_the_scales(mp, tokens):  # noqa: F811
    """With fp32 results entries are those of bf16: multiples of 2^-133 below 2^-126 (half a step off at most), infinities from 2^128 on.
    A scale of 255 is NaN in every type."""
    def q8(codes, scale):
        c = torch.zeros(len(codes), 128, dtype=torch.uint8, device="cuda")
        c[:, 0] = torch.as_tensor(codes, device="cuda")
        return mp.Q8(128, c.view(torch.float8_e4m3fn), torch.full((len(codes), 4), scale, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu))
    positive = np.arange(127, dtype=np.uint8)                  # every code but NaN, in their order
    one = np.full(tokens, 0x38, np.uint8)
    value = torch.from_numpy(positive).view(torch.float8_e4m3fn).float().double().numpy()
    for scale in (0, 1, 2, 5, 6, 10, 200, 246, 247, 248, 254):
        other = 227 if scale < 100 else 27                     # 2^100, 2^-100
        got = values(mp.q8_linear(q8(one, other), q8(positive, scale), dtype=torch.float32)) * 2.0 ** (127.0 - other)
        entry = value * 2.0 ** (scale - 127.0)
        inside = entry < 2.0 ** 128
        off = np.where(entry < 2.0 ** -126, 2.0 ** -134, 0.0)
        assert (np.abs(got - entry)[:, inside] <= off[inside]).all() and np.isinf(got[:, ~inside]).all(), scale
    for dtype in TYPES.values():
        assert torch.isnan(mp.q8_linear(q8(one, 255), q8(positive, 127), dtype=dtype)).all()
        assert torch.isnan(mp.q8_linear(q8(one, 127), q8(positive, 255), dtype=dtype)).all()


def test_layers_that_share_a_step_have_masks_of_their_own(mp):  # noqa: F811
    """Offsets further apart than the step goes, or seeds; the mask is that of the sum of offset and step."""
    x = torch.ones(20, 64, device="cuda")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    masks = []
    layers = [mp.Dropout(0.5, 9, layer << 40, step=step) for layer in range(4)] + [mp.Dropout(0.5, seed, 0, step=step) for seed in (10, 11)]
    for now in range(4):
        step.fill_(now)
        for k, drop in enumerate(layers):
            y = mp.dropout(x, drop)
            masks.append(y != 0)
            seed, offset = (9, k << 40) if k < 4 else (6 + k, 0)
            np.testing.assert_array_equal(values(masks[-1]) != 0, lo.kept(20, 64, 0.5, seed, offset + now))
    for i in range(len(masks)):
        for j in range(i):
            assert not torch.equal(masks[i], masks[j])
    step.fill_(3)
    assert torch.equal(mp.dropout(x, mp.Dropout(0.5, 9, 1, step=step)), mp.dropout(x, mp.Dropout(0.5, 9, 4)))


def test_dropout_of_nearly_everything(mp):  # noqa: F811
    """p next to 1: the threshold is the largest word, and what is kept is divided by 1 - p."""
    x = torch.ones(64, 512, device="cuda")
    for p in (1 - 2.0 ** -12, 1 - 2.0 ** -32, 1 - 2.0 ** -40, 1 - 2.0 ** -53):
        y, keep = values(mp.dropout(x, mp.Dropout(p, 5, 6))), lo.kept(64, 512, p, 5, 6)
        np.testing.assert_array_equal(y, np.where(keep, 1 / (1 - p), 0.0))
