"""GPU parity of the pruned feed-forward block (gated products, norms, 4-bit products) against the 64-bit oracle.

Tolerances are bounds, not fits.  With u = 2^-24 and e the unit roundoff of the storage type, a sum of K products
in fp32 is off by at most (2 K + 64) u sum|a||b| (one rounding per addition, in whatever order and with a factor of two for
matrix cores that align before they add; fp32 operands cut into bf16 parts lose another 2^-20), an elementary function by
16 u of its value and its arguments' error times its slope, and a result by e of itself when it is stored."""
import numpy as np
import pytest

from oracle import block_oracle as bo

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
ROUND = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8 * 1.001, "f16": 2.0 ** -11 * 1.001}
TINY = {"f32": 1e-37, "bf16": 1e-37, "f16": 2.0 ** -24}      # what a stored result may lose below the normal range
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def mp():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2405_02086_amd import binding
    binding.lib()
    return binding


def matrix(rng, rows, cols, dtype, scale=1.0, gap=0):
    """A device matrix whose rows are `gap` elements further apart than they are long, and its values in 64 bits."""
    host = torch.from_numpy(rng.standard_normal((rows, cols + gap)).astype(np.float32) * scale).to(TYPES[dtype])
    return host.to("cuda")[:, :cols], host[:, :cols].double().numpy()


def values(t):
    return t.detach().double().cpu().numpy()


def close(got, want, bound, what):
    got = values(got)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), "%s: %d of %d entries off, the first at %s: %r, not %r (+- %r)" % (
        what, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0], np.broadcast_to(bound, want.shape)[bad][0])


def sum_bound(K, dtype):
    return (2 * K + 64) * U32 + (2.0 ** -20 if dtype == "f32" else 0.0)


def stored(want, dtype):
    return ROUND[dtype] * np.abs(want) + TINY[dtype]


# |act'| <= 1.13 for both smooth activations, and |act''| <= 0.8
SLOPE, CURVE = 1.13, 0.8

SIZES = [(1, 1, 1), (2, 3, 5), (16, 256, 128), (1, 40, 300), (5, 129, 1000), (17, 33, 65), (31, 520, 72), (64, 64, 64), (65, 127, 129),
         (128, 128, 128), (129, 200, 257), (200, 1001, 130), (257, 72, 520), (300, 264, 1032), (520, 512, 640)]


def ff_case(mp, rng, tokens, n, m, dtype, mask_share, joined, gap=0):
    X, x = matrix(rng, tokens, n, dtype, gap=gap)
    if joined:
        W, w = matrix(rng, n, 2 * m, dtype, scale=n ** -0.5, gap=gap)
        Wg, Wu, wg, wu = W[:, :m], W[:, m:], w[:, :m], w[:, m:]
    else:
        (Wg, wg), (Wu, wu) = matrix(rng, n, m, dtype, n ** -0.5, gap), matrix(rng, n, m, dtype, n ** -0.5, gap)
    mask = None
    if mask_share is not None:
        mask = (rng.random(m) < mask_share).astype(np.uint8)
    return X, x, Wg, wg, Wu, wu, mask, None if mask is None else torch.from_numpy(mask).cuda()


def check_forward(mp, rng, tokens, n, m, dtype, act, mask_share=None, joined=False, saved=False, gap=0):
    X, x, Wg, wg, Wu, wu, mask, dmask = ff_case(mp, rng, tokens, n, m, dtype, mask_share, joined, gap)
    H, G, U = bo.gated_ff(x, wg, wu, act, mask)
    c = sum_bound(n, dtype)
    eg, eu = c * (np.abs(x) @ np.abs(wg)), c * (np.abs(x) @ np.abs(wu))
    if mask is not None:
        eg[:, mask == 0] = eu[:, mask == 0] = 0
    a = np.abs(bo.activation(act, G))
    eh = (SLOPE * eg + 16 * U32 * (a + np.abs(G))) * (np.abs(U) + eu) + a * eu
    pad = torch.full((tokens + 1, m + gap + 3), 7.0, dtype=TYPES[dtype], device="cuda")
    out = pad[:tokens, :m]
    g = u = None
    if saved:
        g, u = torch.full((2, tokens, m), 7.0, dtype=TYPES[dtype], device="cuda")
    ws = mp.Workspace(mp.gated_ff_workspace_bytes(tokens, n, m, TYPES[dtype]))
    ws.buf.fill_(255)
    got = mp.gated_ff(X, Wg, Wu, act=act, mask=dmask, H=out, g_out=g, u_out=u, workspace=ws)
    torch.cuda.synchronize()
    assert got.data_ptr() == out.data_ptr()
    close(out, H, eh + stored(H, dtype), "H")
    assert (pad[tokens:] == 7).all() and (pad[:, m:] == 7).all(), "written outside of H"
    if saved:
        close(g, G, eg + stored(G, dtype), "G")
        close(u, U, eu + stored(U, dtype), "U")


def check_backward(mp, rng, tokens, n, m, dtype, act, mask_share=None, joined=False, saved=False, gap=0, need_dx=True, need_dw=True):
    X, x, Wg, wg, Wu, wu, mask, dmask = ff_case(mp, rng, tokens, n, m, dtype, mask_share, joined, gap)
    dH, dh = matrix(rng, tokens, m, dtype, gap=gap)
    G = U = g = u = None
    if saved:
        (G, g), (U, u) = matrix(rng, tokens, m, dtype, gap=gap), matrix(rng, tokens, m, dtype, gap=gap)
    dX, dWg, dWu, dG, dU = bo.gated_ff_backward(dh, x, wg, wu, act, mask, g, u)
    # errors of dG and dU: of G and U where they are computed, of the functions, of one rounding to the storage type
    c = sum_bound(n, dtype)
    g0, u0 = (g, u) if saved else (x @ wg, x @ wu)
    eg, eu = (0, 0) if saved else (c * (np.abs(x) @ np.abs(wg)), c * (np.abs(x) @ np.abs(wu)))
    slope, a = np.abs(bo.activation_slope(act, g0)), np.abs(bo.activation(act, g0))
    if act == "relu":       # the slope jumps where the sign of G is in doubt
        jump = (np.abs(g0) <= eg).astype(float)
        e_slope = jump
    else:
        e_slope = CURVE * eg + 32 * U32 * (1 + np.abs(g0))
    e_dg = np.abs(dh) * (slope * eu + (np.abs(u0) + eu) * e_slope)
    e_du = np.abs(dh) * (SLOPE * eg + 16 * U32 * (a + np.abs(g0)))
    e_dg = e_dg + stored(dG, dtype) + ROUND[dtype] * e_dg
    e_du = e_du + stored(dU, dtype) + ROUND[dtype] * e_du
    if mask is not None:
        e_dg[:, mask == 0] = e_du[:, mask == 0] = 0
    kx, kw = sum_bound(2 * m, dtype), sum_bound(tokens, dtype)
    wg_, wu_, x_ = np.abs(wg), np.abs(wu), np.abs(x)
    ax = (np.abs(dG) + e_dg) @ wg_.T + (np.abs(dU) + e_du) @ wu_.T
    bx = e_dg @ wg_.T + e_du @ wu_.T + kx * ax
    bg = x_.T @ e_dg + kw * (x_.T @ (np.abs(dG) + e_dg))
    bu = x_.T @ e_du + kw * (x_.T @ (np.abs(dU) + e_du))
    ws = mp.Workspace(mp.gated_ff_workspace_bytes(tokens, n, m, TYPES[dtype], True))
    ws.buf.fill_(255)
    pads = [torch.full((r + 1, k + gap + 3), 7.0, dtype=TYPES[dtype], device="cuda") for r, k in ((tokens, n), (n, m), (n, m))]
    outs = [p[:r, :k] for p, (r, k) in zip(pads, ((tokens, n), (n, m), (n, m)))]
    got = mp.gated_ff_backward(dH, X, Wg, Wu, act=act, mask=dmask, G=G, U=U, dX=outs[0], dWg=outs[1], dWu=outs[2], workspace=ws,
                               need_dx=need_dx, need_dw=need_dw)
    torch.cuda.synchronize()
    if need_dx:
        close(got[0], dX, bx + stored(dX, dtype), "dX")
    if need_dw:
        close(got[1], dWg, bg + stored(dWg, dtype), "dWg")
        close(got[2], dWu, bu + stored(dWu, dtype), "dWu")
        if mask is not None:
            assert (got[1][:, dmask == 0] == 0).all() and (got[2][:, dmask == 0] == 0).all()
    assert (got[0] is None) == (not need_dx) and (got[1] is None) == (not need_dw)
    for p, (r, k) in zip(pads, ((tokens, n), (n, m), (n, m))):
        assert (p[r:] == 7).all() and (p[:, k:] == 7).all(), "written outside"


ACTS = ["silu", "gelu", "relu"]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("i", range(len(SIZES)))
def test_gated_ff_forward(mp, i, dtype):
    tokens, n, m = SIZES[i]
    rng = np.random.default_rng(100 + i)
    check_forward(mp, rng, tokens, n, m, dtype, ACTS[i % 3])
    check_forward(mp, rng, tokens, n, m, dtype, ACTS[(i + 1) % 3], mask_share=0.4, joined=i % 2 == 0, saved=i % 4 == 1)
    check_forward(mp, rng, tokens, n, m, dtype, ACTS[(i + 2) % 3], saved=True, gap=3 if i % 2 else 8)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("i", range(len(SIZES)))
def test_gated_ff_backward(mp, i, dtype):
    tokens, n, m = SIZES[i]
    rng = np.random.default_rng(200 + i)
    check_backward(mp, rng, tokens, n, m, dtype, ACTS[i % 3])
    check_backward(mp, rng, tokens, n, m, dtype, ACTS[(i + 1) % 3], mask_share=0.4, joined=i % 2 == 0, saved=i % 4 == 1)
    check_backward(mp, rng, tokens, n, m, dtype, ACTS[(i + 2) % 3], saved=True, gap=3 if i % 2 else 8, need_dx=i % 3 != 0, need_dw=i % 3 != 1)


@pytest.mark.parametrize("share", [0.0, 0.02, 0.97, 1.0])
@pytest.mark.parametrize("tokens", [1, 40, 150])
def test_gated_ff_masks(mp, share, tokens):
    """Nothing kept, nearly nothing, nearly everything, everything."""
    rng = np.random.default_rng(7)
    for dtype, n, m in (("bf16", 136, 520), ("f32", 40, 333), ("f16", 201, 77)):
        check_forward(mp, rng, tokens, n, m, dtype, "silu", mask_share=share)
        check_backward(mp, rng, tokens, n, m, dtype, "gelu", mask_share=share)
        check_backward(mp, rng, tokens, n, m, dtype, "silu", mask_share=share, saved=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens", [3, 70, 200])
def test_gated_ff_pruned_channels_ignore_what_they_hold(mp, dtype, tokens):
    """NaN and infinities in the weights and gradients of pruned channels reach nothing."""
    rng = np.random.default_rng(8)
    n, m = 72, 264
    X, x, Wg, wg, Wu, wu, mask, dmask = ff_case(mp, rng, tokens, n, m, dtype, 0.5, False)
    dH, dh = matrix(rng, tokens, m, dtype)
    G, U = torch.empty(2, tokens, m, dtype=TYPES[dtype], device="cuda")
    clean = mp.gated_ff(X, Wg, Wu, mask=dmask, g_out=G, u_out=U)
    grads = mp.gated_ff_backward(dH, X, Wg, Wu, mask=dmask)
    pruned = dmask == 0
    Wg, Wu, dH, G, U = Wg.clone(), Wu.clone(), dH.clone(), G.clone(), U.clone()
    Wg[:, pruned] = float("nan")
    Wu[:, pruned] = float("inf")
    dH[:, pruned] = float("-inf")
    G[:, pruned] = U[:, pruned] = float("nan")
    dirty = mp.gated_ff(X, Wg, Wu, mask=dmask)
    assert torch.equal(clean, dirty)
    for a, b in zip(grads, mp.gated_ff_backward(dH, X, Wg, Wu, mask=dmask)):
        assert torch.equal(a, b)
    for a in mp.gated_ff_backward(dH, X, Wg, Wu, mask=dmask, G=G, U=U):
        assert torch.isfinite(a).all()


def test_gated_ff_non_finite_inputs_stay_in_their_rows(mp):
    rng = np.random.default_rng(9)
    for dtype in ("f32", "bf16"):
        for tokens in (20, 150):
            X, _ = matrix(rng, tokens, 96, dtype)
            Wg, _ = matrix(rng, 96, 136, dtype, 0.1)
            Wu, _ = matrix(rng, 96, 136, dtype, 0.1)
            clean = mp.gated_ff(X, Wg, Wu)
            X = X.clone()
            X[3, 5] = float("nan")
            X[7, 9] = float("inf")
            dirty = mp.gated_ff(X, Wg, Wu)
            assert torch.isnan(dirty[3]).all()
            assert not torch.isfinite(dirty[7]).any()
            rows = [t for t in range(tokens) if t not in (3, 7)]
            assert torch.equal(clean[rows], dirty[rows])


def test_gated_ff_without_tokens(mp):
    for dtype in TYPES.values():
        X = torch.empty(0, 24, dtype=dtype, device="cuda")
        W = torch.ones(24, 40, dtype=dtype, device="cuda")
        assert mp.gated_ff(X, W, W).shape == (0, 40)
        dX, dWg, dWu = mp.gated_ff_backward(torch.empty(0, 40, dtype=dtype, device="cuda"), X, W, W)
        assert dX.shape == (0, 24) and not dWg.any() and not dWu.any() and dWg.shape == (24, 40)


@pytest.mark.parametrize("tokens,n,m", [(1, 4096, 2048), (40, 2048, 1024), (700, 1536, 1280), (2048, 1024, 1536)])
def test_gated_ff_larger(mp, tokens, n, m):
    rng = np.random.default_rng(10)
    check_forward(mp, rng, tokens, n, m, "bf16", "silu", mask_share=0.5 if tokens > 1 else None, saved=True)
    check_backward(mp, rng, tokens, n, m, "bf16", "gelu", mask_share=0.5)
    check_backward(mp, rng, tokens, n, m, "f16", "silu", saved=True)


def test_gated_ff_same_bits_every_time_and_on_another_stream(mp):
    rng = np.random.default_rng(11)
    for tokens, n, m in ((1, 2000, 520), (30, 2000, 520), (300, 1000, 700)):
        X, x, Wg, wg, Wu, wu, mask, dmask = ff_case(mp, rng, tokens, n, m, "bf16", 0.5, False)
        dH, _ = matrix(rng, tokens, m, "bf16")
        torch.cuda.synchronize()
        once = [mp.gated_ff(X, Wg, Wu), *mp.gated_ff_backward(dH, X, Wg, Wu, mask=dmask)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = [mp.gated_ff(X, Wg, Wu), *mp.gated_ff_backward(dH, X, Wg, Wu, mask=dmask)]
        side.synchronize()
        for a, b in zip(once, again):
            assert torch.equal(a, b)


# ---------------------------------------------------------------- norms

NORM_SIZES = [(1, 1), (3, 5), (2, 63), (7, 64), (5, 512), (9, 513), (4, 1000), (3, 1025), (6, 2048), (5, 3001), (3, 4096), (2, 5001), (2, 8200),
              (3, 16384), (2, 16390), (1300, 40), (700, 3003), (2100, 256)]


def norm_case(rng, tokens, n, dtype, token_gate, gap):
    x = matrix(rng, tokens, n, dtype, 2.0, gap)
    b = matrix(rng, tokens, n, dtype, 0.7, gap)
    w = [matrix(rng, 1, n, dtype) for _ in range(2)]
    gate = matrix(rng, tokens, n, dtype, gap=gap) if token_gate else tuple(a[0] for a in matrix(rng, 1, n, dtype))
    return x, b, (w[0][0][0], w[0][1][0]), gate, (w[1][0][0], w[1][1][0])


def norm_forward_bounds(x, b, w_post, gate, w_pre, scale, eps, dtype):
    """r, y and the bounds: a mean of squares is off by (n + 8) u of itself, its root by half of that."""
    r, y = bo.block_norm(x, b, w_post, gate, w_pre, scale, eps)
    n = x.shape[1]
    k = (n + 32) * U32
    er = np.zeros_like(r) if b is None else k * np.abs(r - x) + 4 * U32 * (np.abs(x) + np.abs(r))
    ey = None
    if y is not None:
        # the root moves by the error of r's mean square, at most max|er| over rms
        s = bo.rms(r, eps)
        ey = np.abs(w_pre) * (er / s) + np.abs(y) * (k + np.sqrt((er * er).mean(1, keepdims=True)) / s)
    return r, y, er, ey


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("i", range(len(NORM_SIZES)))
def test_block_norm(mp, i, dtype):
    tokens, n = NORM_SIZES[i]
    rng = np.random.default_rng(300 + i)
    for token_gate, gap in ((False, 0), (True, 5 if i % 2 else 0)):
        (X, x), (B, b), (WP, wp), (G, g), (WQ, wq) = norm_case(rng, tokens, n, dtype, token_gate, gap)
        for parts in ("both", "pre", "post"):
            kw = dict(scale=0.6, eps=1e-5)
            blk = {} if parts == "pre" else dict(b=B, w_post=WP, gate=G)
            ref = {} if parts == "pre" else dict(b=b, w_post=wp, gate=g)
            pre = None if parts == "post" else WQ
            r, y, er, ey = norm_forward_bounds(x, ref.get("b"), ref.get("w_post"), ref.get("gate"), None if pre is None else wq, 0.6, 1e-5, dtype)
            R, Y = mp.block_norm(X, w_pre=pre, **blk, **kw)
            torch.cuda.synchronize()
            if parts == "pre":
                assert R is X
            else:
                close(R, r, er + stored(r, dtype), "r")
            if pre is None:
                assert Y is None
            else:
                close(Y, y, ey + stored(y, dtype), "y")
    # in place: r over x, y over b
    want_r, want_y = mp.block_norm(X, B, WP, G, WQ, scale=0.6)
    Xc, Bc = X.clone(), B.clone()
    mp.block_norm(Xc, Bc, WP, G, WQ, scale=0.6, r=Xc, y=Bc)
    assert torch.equal(Xc, want_r) and torch.equal(Bc, want_y)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("i", range(len(NORM_SIZES)))
def test_block_norm_backward(mp, i, dtype):
    tokens, n = NORM_SIZES[i]
    rng = np.random.default_rng(400 + i)
    eps, scale = 1e-5, 0.6
    for token_gate, gap in ((False, 0), (True, 5 if i % 2 else 0)):
        (R, r), (B, b), (WP, wp), (G, g), (WQ, wq) = norm_case(rng, tokens, n, dtype, token_gate, gap)
        (DR, dr), (DY, dy) = matrix(rng, tokens, n, dtype, gap=gap), matrix(rng, tokens, n, dtype, gap=gap)
        for parts in ("both", "pre", "post", "no dr"):
            blk = {} if parts == "pre" else dict(b=B, w_post=WP, gate=G)
            ref = {} if parts == "pre" else dict(b=b, w_post=wp, gate=g)
            pre, wpre = (None, None) if parts == "post" else (WQ, wq)
            DRp, drp = (None, None) if parts == "no dr" else (DR, dr)
            dx, db, dwp, dg, dwq = bo.block_norm_backward(drp, dy, r, w_pre=wpre, scale=scale, eps=eps, **ref)
            ws = mp.Workspace(mp.block_norm_workspace_bytes(tokens, n))
            ws.buf.fill_(255)
            got = mp.block_norm_backward(DRp, None if pre is None else DY, R, w_pre=pre, scale=scale, eps=eps, workspace=ws, **blk)
            torch.cuda.synchronize()
            # every sum over a row of n terms is off by (n + 32) u of the sum of its terms' magnitudes, every elementwise
            # result by a few u of its terms
            k = (n + 64) * U32
            sr, sb = bo.rms(r, eps), bo.rms(b, eps)
            e = np.zeros_like(r) if wpre is None else np.abs(wq * dy)
            spread = np.abs(r) / sr * (np.abs(r) / sr * e).mean(1, keepdims=True) / sr
            mag_x = np.abs(drp if drp is not None else 0) + e / sr + spread
            ex = k * mag_x
            close(got[0], dx, ex + stored(dx, dtype), "dx")
            if pre is None:
                assert got[4] is None
            else:
                t = np.abs(dy * (r / sr))
                close(got[4], dwq, (k + (tokens + 16) * U32) * t.sum(0) + 1e-37, "dw_pre")
            if parts == "pre":
                assert got[1] is None and got[2] is None and got[3] is None
                continue
            f = np.abs(scale * g * wp)
            bh = np.abs(b) / sb
            fx = f * mag_x
            close(got[1], db, 4 * k * (fx / sb + bh * (bh * fx).mean(1, keepdims=True) / sb) + stored(db, dtype), "db")
            close(got[2], dwp, (4 * k + (tokens + 16) * U32) * (np.abs(scale * g) * mag_x * bh).sum(0) + 1e-37, "dw_post")
            tg = np.abs(scale * wp) * mag_x * bh
            if token_gate:
                close(got[3], dg, 4 * k * tg + stored(dg, dtype), "dgate")
            else:
                close(got[3], dg, (4 * k + (tokens + 16) * U32) * tg.sum(0) + 1e-37, "dgate")


def test_block_norm_in_place_gradients_and_zero_rows(mp):
    rng = np.random.default_rng(12)
    for n in (100, 1500, 17000):
        (R, r), (B, b), (WP, wp), (G, g), (WQ, wq) = norm_case(rng, 6, n, "bf16", False, 0)
        (DR, dr), (DY, dy) = matrix(rng, 6, n, "bf16"), matrix(rng, 6, n, "bf16")
        R, B = R.clone(), B.clone()
        R[2] = 0
        B[3] = 0
        want = mp.block_norm_backward(DR, DY, R, B, WP, G, WQ)
        assert all(torch.isfinite(t).all() for t in want)
        DRc, Bc = DR.clone(), B.clone()
        got = mp.block_norm_backward(DRc, DY, R, Bc, WP, G, WQ, dx=DRc, db=Bc)
        for a, c in zip(want, got):
            assert torch.equal(a, c)
        r2, y2 = mp.block_norm(torch.zeros(2, n, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, n, dtype=torch.bfloat16, device="cuda"), WP, G, WQ)
        assert not r2.any() and not y2.any()


def test_block_norm_without_tokens(mp):
    e = torch.empty(0, 48, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(48, dtype=torch.bfloat16, device="cuda")
    r, y = mp.block_norm(e, e, w, w, w)
    assert r.shape == y.shape == (0, 48)
    dx, db, dwp, dg, dwq = mp.block_norm_backward(e, e, e, e, w, w, w)
    assert dx.shape == (0, 48) and not dwp.any() and not dg.any() and not dwq.any()


# ---------------------------------------------------------------- 4-bit weights

W4_SIZES = [(1, 1), (5, 3), (32, 16), (100, 33), (128, 16), (129, 17), (300, 200), (1000, 250), (2048, 64), (257, 1040)]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_w4_pack(mp, dtype, group):
    rng = np.random.default_rng(13)
    for n, m in [(1, 1), (5, 3), (130, 33), (300, 17)]:
        W, w = matrix(rng, n, m, dtype, 0.05, gap=3)
        if m > 2:
            W[:, 1] = 0           # a pruned column
            w[:, 1] = 0
        codes, scales = bo.w4_quantise(w, group)
        want, want_scales = bo.w4_layout(codes, scales, group)
        packed = mp.w4_pack(W, group)
        torch.cuda.synchronize()
        assert np.array_equal(packed.codes.cpu().numpy().reshape(want.shape), want)
        assert np.array_equal(packed.scales.float().cpu().numpy().reshape(want_scales.shape), want_scales)


def w4_matrix(mp, rng, n, m, group):
    W, w = matrix(rng, n, m, "f32", n ** -0.5)
    codes, scales = bo.w4_quantise(w, group)
    return mp.w4_pack(W, group), bo.w4_values(codes, scales, group)


@pytest.mark.parametrize("tokens", [1, 2, 16, 17, 32, 33, 64, 65, 150])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_w4_products(mp, dtype, tokens):
    rng = np.random.default_rng(14 + tokens)
    for i, (n, m) in enumerate(W4_SIZES):
        group = (32, 64, 128)[(i + tokens) % 3]
        act = ACTS[i % 3]
        gap = (0, 3, 8)[i % 3]
        X, x = matrix(rng, tokens, n, dtype, gap=gap)
        Wg, wg = w4_matrix(mp, rng, n, m, group)
        Wu, wu = w4_matrix(mp, rng, n, m, group)
        c = sum_bound(n, dtype)
        g, u = x @ wg, x @ wu
        eg, eu = c * (np.abs(x) @ np.abs(wg)), c * (np.abs(x) @ np.abs(wu))
        pad = torch.full((tokens + 1, m + 3), 7.0, dtype=TYPES[dtype], device="cuda")
        mp.w4_matvec(X, Wg, y=pad[:tokens, :m])
        torch.cuda.synchronize()
        close(pad[:tokens, :m], g, eg + stored(g, dtype), "y")
        assert (pad[tokens:] == 7).all() and (pad[:, m:] == 7).all()
        a = np.abs(bo.activation(act, g))
        h = bo.activation(act, g) * u
        eh = (SLOPE * eg + 16 * U32 * (a + np.abs(g))) * (np.abs(u) + eu) + a * eu
        close(mp.w4_gated_matvec(X, Wg, Wu, act=act), h, eh + stored(h, dtype), "h")


def test_w4_larger_and_no_tokens(mp):
    rng = np.random.default_rng(15)
    for n, m, group, dtype, tokens in ((4096, 1024, 128, "bf16", 1), (8192, 256, 32, "f16", 16), (1000, 4100, 64, "bf16", 5)):
        W, w = w4_matrix(mp, rng, n, m, group)
        X, x = matrix(rng, tokens, n, dtype)
        y = x @ w
        close(mp.w4_matvec(X, W), y, sum_bound(n, dtype) * (np.abs(x) @ np.abs(w)) + stored(y, dtype), "y")
        assert torch.equal(mp.w4_matvec(X, W), mp.w4_matvec(X, W))
    assert mp.w4_matvec(torch.empty(0, 1000, device="cuda"), W).shape == (0, 4100)


# ---------------------------------------------------------------- routes, larger sizes, graphs, the example

def blocks_close(got, want, e, what, side=64):
    """Every side x side block of a result is as near the 64-bit one as two roundings of its entries allow (each at most e
    of an entry or of the terms it is summed from, whose errors add up as a norm): a tile that went wrong stands out."""
    got, want = got.double(), want
    rows, cols = want.shape
    pad = (-rows % side, -cols % side)
    def norms(t):
        t = torch.nn.functional.pad(t, (0, pad[1], 0, pad[0]))
        return t.view(t.shape[0] // side, side, t.shape[1] // side, side).square().sum((1, 3)).sqrt()
    off, size = norms(got - want), norms(want)
    bad = ~(off <= 4 * e * size + 1e-30)
    assert not bad.any(), "%s: blocks off: %s" % (what, bad.nonzero()[:5].tolist())


def exact_block(X, Wg, Wu, dH, act, mask):
    x, wg, wu = X.double(), Wg.double(), Wu.double()
    k = mask.double() if mask is not None else 1.0
    g, u = x @ wg, x @ wu
    if act == "silu":
        s = torch.sigmoid(g)
        a, slope = g * s, s * (1 + g * (1 - s))
    else:
        a, slope = torch.relu(g), (g > 0).double()
    dg, du = dH.double() * u * slope * k, dH.double() * a * k
    return {"H": a * u * k, "G": g * k, "U": u * k, "dX": dg @ (wg * k).t() + du @ (wu * k).t(), "dWg": x.t() @ dg, "dWu": x.t() @ du}


# sizes whose products take: whole turns and a rest of smaller tiles (packed or not), shares of the sum in every kind of tile, ...
ROUTES = [(4200, 512, 4200, 0, {"kind": 0, "parts": True}), (2100, 2056, 8200, 1, {"kind": 0, "parts": True, "packed": True}),
          (2304, 2048, 4400, 2, {"kind": 0, "packed": True}), (1100, 2048, 9000, 3, {"kind": 0, "parts": True}),
          (300, 8192, 64, 1, {"kind": 1}), (1000, 1000, 10000, 2, {"kind": 0, "shares": 16}), (3617, 1032, 4096, 1, {"packed": True}), (2048, 1024, 1536, 0, {"kind": 1, "shares": 1}),
          (1024, 4096, 512, 0, {"kind": 1, "low": True, "shares": 2}), (514, 4096, 2048, 1, {"kind": 1, "low": False, "shares": 1}),
          (1300, 776, 2056, 2, {"kind": 1, "low": True, "shares": 1}), (310, 824, 6432, 2, {"kind": 1, "low": False, "shares": 8}),
          (2500, 800, 2400, 3, {"kind": 1, "low": True, "shares": 1})]


@pytest.mark.parametrize("case", range(len(ROUTES)))
@pytest.mark.parametrize("masked", [False, True])
def test_gated_ff_routes(mp, case, masked):
    tokens, n, m, product, route = ROUTES[case]
    dtype = "bf16" if case % 2 else "f16"
    got = mp.gated_ff_route(TYPES[dtype], product, tokens, n, m)
    assert {k: got[k] for k in route} == route
    gen = torch.Generator(device="cuda")
    gen.manual_seed(40 + case)
    new = lambda r, c, s=1.0: (torch.randn(r, c, generator=gen, device="cuda") * s).to(TYPES[dtype])  # noqa: E731
    X, Wg, Wu, dH = new(tokens, n), new(n, m, n ** -0.5), new(n, m, n ** -0.5), new(tokens, m)
    mask = (torch.rand(m, generator=gen, device="cuda") < 0.55).to(torch.uint8) if masked else None
    act = ("silu", "relu")[case % 2] if case != 1 else "silu"
    want = exact_block(X, Wg, Wu, dH, act, mask)
    G, U = torch.empty(2, tokens, m, dtype=TYPES[dtype], device="cuda")
    H = mp.gated_ff(X, Wg, Wu, act=act, mask=mask, g_out=G, u_out=U)
    for name, t in (("H", H), ("G", G), ("U", U)):
        blocks_close(t, want[name], ROUND[dtype], name)
    # a relu whose argument rounds to the other side of 0 changes whole entries of its gradient, but only where both are tiny
    for name, t in zip(("dX", "dWg", "dWu"), mp.gated_ff_backward(dH, X, Wg, Wu, act=act, mask=mask)):
        blocks_close(t, want[name], ROUND[dtype], name)


def test_gated_ff_fp32_larger(mp):
    for tokens, n, m in ((700, 1000, 1100), (40, 3000, 700), (1500, 264, 2056)):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(tokens)
        new = lambda r, c, s=1.0: torch.randn(r, c, generator=gen, device="cuda") * s  # noqa: E731
        X, Wg, Wu, dH = new(tokens, n), new(n, m, n ** -0.5), new(n, m, n ** -0.5), new(tokens, m)
        for mask in (None, (torch.rand(m, generator=gen, device="cuda") < 0.5).to(torch.uint8)):
            want = exact_block(X, Wg, Wu, dH, "silu", mask)
            # fp32 sums of up to 4000 terms: sqrt(4000) roundings of 2^-24 in a random walk, and the function's 16
            e = 100 * U32
            blocks_close(mp.gated_ff(X, Wg, Wu, mask=mask), want["H"], e, "H")
            for name, t in zip(("dX", "dWg", "dWu"), mp.gated_ff_backward(dH, X, Wg, Wu, mask=mask)):
                blocks_close(t, want[name], e, name)


def test_gated_ff_fp32_few_tokens_packed(mp):
    tokens, n, m = 9, 4096, 12004
    assert mp.gated_ff_route(torch.float32, 1, tokens, n, m)["packed"] and mp.gated_ff_route(torch.float32, 1, tokens, n, m)["kind"] == 3
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    new = lambda r, c, s=1.0: torch.randn(r, c, generator=gen, device="cuda") * s  # noqa: E731
    X, Wg, Wu, dH = new(tokens, n), new(n, m, n ** -0.5), new(n, m, n ** -0.5), new(tokens, m)
    for keep in (0.0, 0.4, 1.0):
        mask = (torch.rand(m, generator=gen, device="cuda") < keep).to(torch.uint8)
        got = mp.gated_ff_backward(dH, X, Wg, Wu, mask=mask)
        if not keep:
            assert not any(t.any() for t in got)
            continue
        want = exact_block(X, Wg, Wu, dH, "silu", mask)
        for name, t in zip(("dX", "dWg", "dWu"), got):
            blocks_close(t, want[name], 100 * U32, name)


def test_block_calls_can_be_captured_in_a_hip_graph(mp):
    rng = np.random.default_rng(16)
    for tokens, n, m, dtype in ((1, 2000, 520, "bf16"), (300, 700, 1000, "bf16"), (20, 300, 200, "f32"), (2100, 1032, 4168, "f16")):
        X, x, Wg, wg, Wu, wu, mask, dmask = ff_case(mp, rng, tokens, n, m, dtype, 0.5, False)
        dH, _ = matrix(rng, tokens, m, dtype)
        w = torch.ones(n, dtype=TYPES[dtype], device="cuda")
        packed = mp.w4_pack(Wg)
        H, h4 = torch.empty_like(dH), torch.empty_like(dH)
        outs = [torch.empty_like(X), torch.empty_like(Wg), torch.empty_like(Wu)]
        r, y = torch.empty_like(X), torch.empty_like(X)
        ws = mp.Workspace(mp.gated_ff_workspace_bytes(tokens, n, m, TYPES[dtype], True))
        wf = mp.Workspace(mp.gated_ff_workspace_bytes(tokens, n, m, TYPES[dtype]))

        def calls():
            mp.gated_ff(X, Wg, Wu, mask=dmask, H=H, workspace=wf)
            mp.gated_ff_backward(dH, X, Wg, Wu, mask=dmask, dX=outs[0], dWg=outs[1], dWu=outs[2], workspace=ws)
            mp.block_norm(X, X, w, w, w, r=r, y=y)
            mp.w4_gated_matvec(X, packed, packed, h=h4)

        calls()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls()
        for turn in range(3):
            X.copy_(matrix(rng, tokens, n, dtype)[0])
            calls()
            want = [t.clone() for t in (H, *outs, r, y, h4)]
            for t in (H, *outs, r, y, h4):
                t.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(want, (H, *outs, r, y, h4)):
                assert torch.equal(a, b)


def test_the_example_learns_prunes_and_answers_in_four_bits(mp):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "pruned_block.py")
    spec = importlib.util.spec_from_file_location("pruned_block", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    out = example.main()
    assert out["last_loss"] < 0.75 * out["first_loss"]
    assert 0 < out["kept"] < out["channels"]
    assert out["four_bit_error"] < 0.2


# ---------------------------------------------------------------- lightly pruned blocks whose channels are packed

FILLS = [("bf16", 1024, 1032, 4096, 1), ("bf16", 1024, 1032, 4096, 3), ("f16", 1024, 1032, 4095, 1), ("bf16", 512, 2048, 6144, 7),
         ("f32", 256, 512, 4096, 1), ("f32", 256, 512, 6144, 3)]


@pytest.mark.parametrize("saved", [False, True])
@pytest.mark.parametrize("case", range(len(FILLS)))
def test_packed_channels_are_filled_up_with_zeros(mp, case, saved):
    """Only the first few channels are pruned, so that the kept ones end inside a piece behind a full last segment of columns.
    The workspace holds NaN: what is summed over and not written shows."""
    dtype, tokens, n, m, pruned = FILLS[case]
    assert mp.gated_ff_route(TYPES[dtype], 1, tokens, n, m)["packed"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(60 + case)
    new = lambda r, c, s=1.0: (torch.randn(r, c, generator=gen, device="cuda") * s).to(TYPES[dtype])  # noqa: E731
    X, Wg, Wu, dH = new(tokens, n), new(n, m, n ** -0.5), new(n, m, n ** -0.5), new(tokens, m)
    mask = torch.ones(m, dtype=torch.uint8, device="cuda")
    mask[:pruned] = 0
    want = exact_block(X, Wg, Wu, dH, "silu", mask)
    G = U = None
    if saved:
        G, U = want["G"].to(TYPES[dtype]), want["U"].to(TYPES[dtype])
    ws = mp.Workspace(mp.gated_ff_workspace_bytes(tokens, n, m, TYPES[dtype], True))
    ws.buf.fill_(255)
    # two roundings (dG and dU, the result), saved pre-activations a third; fp32: sums of 2 m terms in a random walk
    e = 120 * U32 if dtype == "f32" else 1.5 * ROUND[dtype]
    for name, t in zip(("dX", "dWg", "dWu"), mp.gated_ff_backward(dH, X, Wg, Wu, mask=mask, G=G, U=U, workspace=ws)):
        assert torch.isfinite(t).all(), name
        blocks_close(t, want[name], e, name)


def test_block_norm_without_tokens_reads_nothing(mp):
    """Sums over no tokens are zeros whatever the vectors hold, and the gate need not be there."""
    import ctypes
    for dtype in TYPES.values():
        e = torch.empty(0, 72, dtype=dtype, device="cuda")
        bad = torch.full((72,), float("nan"), dtype=dtype, device="cuda")
        for t in mp.block_norm_backward(e, e, e, e, bad, bad, bad)[2:]:
            assert not t.any()
        ws = mp.Workspace(mp.block_norm_workspace_bytes(0, 72))
        sums = torch.full((3, 72), 7.0, device="cuda")
        block = mp.NormBlock(0, 72, None, 0, bad.data_ptr(), None, 0, bad.data_ptr(), 1.0, 1e-6)
        st = mp.lib().block_norm_backward(mp._storage(dtype), ctypes.byref(block), None, 0, None, 0, None, 0, None, 0, None, 0,
                                          sums[0].data_ptr(), sums[1].data_ptr(), 0, sums[2].data_ptr(), ws.buf.data_ptr(), ws.nbytes,
                                          torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert st == 0 and not sums.any()


def test_block_norm_without_a_block_does_not_use_its_gate(mp):
    """w_post = NULL: b and gate may be anything, at any address."""
    import ctypes
    rng = np.random.default_rng(18)
    for n in (40, 3000, 9000, 17000):
        X, _ = matrix(rng, 5, n, "bf16")
        DY, _ = matrix(rng, 5, n, "bf16")
        w = matrix(rng, 1, n, "bf16")[0][0]
        unused = torch.full((2 * n + 16,), 255, dtype=torch.uint8, device="cuda")
        _, want = mp.block_norm(X, w_pre=w)
        dx, _, _, _, dw = mp.block_norm_backward(None, DY, X, w_pre=w)
        ws = mp.Workspace(mp.block_norm_workspace_bytes(5, n))
        block = mp.NormBlock(5, n, None, 0, None, unused.data_ptr() + 1, 0, w.data_ptr(), 1.0, 1e-6)
        y, dx2, dw2 = torch.empty_like(X), torch.empty_like(X), torch.empty_like(dw)
        stream = torch.cuda.current_stream().cuda_stream
        assert mp.lib().block_norm_forward(1, ctypes.byref(block), X.data_ptr(), n, None, 0, y.data_ptr(), n, stream) == 0
        assert mp.lib().block_norm_backward(1, ctypes.byref(block), X.data_ptr(), n, None, 0, DY.data_ptr(), n, dx2.data_ptr(), n, None, 0,
                                            None, None, 0, dw2.data_ptr(), ws.buf.data_ptr(), ws.nbytes, stream) == 0
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(dx, dx2) and torch.equal(dw, dw2)


def pools(tensors):
    """The streams whose memory the tensors lie in."""
    at = {}
    for seg in torch.cuda.memory_snapshot():
        for t in tensors:
            if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
                at[t.data_ptr()] = seg["stream"]
    return [at[t.data_ptr()] for t in tensors]


def test_calls_given_a_stream_allocate_on_it(mp, monkeypatch):
    """Every call with stream=, results and scratch alike, and a norm that is read back."""
    side = torch.cuda.Stream()
    scratch = []
    init = mp.Workspace.__init__

    def noted(self, *args, **kw):
        init(self, *args, **kw)
        scratch.append(self.buf)

    monkeypatch.setattr(mp.Workspace, "__init__", noted)
    rng = np.random.default_rng(19)
    X, Wg = matrix(rng, 20, 72, "bf16")[0], matrix(rng, 72, 136, "bf16")[0]
    dH, w, Y = matrix(rng, 20, 136, "bf16")[0], matrix(rng, 1, 72, "bf16")[0][0], matrix(rng, 40, 24, "f32")[0]
    cube, weights = matrix(rng, 6, 20, "f32")[0].view(6, 4, 5), torch.ones(24, device="cuda")
    torch.cuda.synchronize()
    kw = dict(stream=side)
    packed = mp.w4_pack(Wg, **kw)
    H = mp.gated_ff(X, Wg, Wg, **kw)
    outs = [packed.codes, packed.scales, H, *mp.gated_ff_backward(dH, X, Wg, Wg, **kw), *mp.block_norm(X, X, w, w, w, **kw),
            *mp.block_norm_backward(None, X, X, X, w, w, w, **kw), *mp.block_norm_backward(None, X, X, X, w, X, w, **kw),
            mp.w4_matvec(X, packed, **kw), mp.w4_gated_matvec(X, packed, packed, **kw),
            mp.bilevel_proj_l1inf(Y, 1.0, **kw), mp.bilevel_proj_pq(2, 1, Y, 1.0, **kw), mp.bilevel_proj_stored(X, 1.0, "inf", **kw),
            mp.bilevel_proj_weighted(Y, 1.0, 2, weights, **kw), mp.trilevel_proj_l1infinf(cube, 1.0, **kw),
            mp.trilevel_proj_stored(cube, 1.0, **kw), *mp.bilevel_proj_batch([Y, Y], [1.0, 2.0], 2, **kw),
            mp.multilevel_proj(cube, [2, "inf"], 1.0, **kw), mp.multilevel_proj_stored(cube, [2, "inf"], 1.0, **kw),
            mp.multilevel_proj_weighted(cube, [2, "inf"], 1.0, weights[:6], **kw)]
    norm = mp.norm_l1q(Y, "l12", **kw)
    assert abs(norm - float(Y.double().norm(dim=0).sum())) < 1e-4 * norm
    assert len(scratch) > 10
    assert set(pools(outs + scratch)) == {side.cuda_stream}
    torch.cuda.synchronize()
    assert torch.equal(H, mp.gated_ff(X, Wg, Wg))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 40, 1000, 17000])
def test_block_norm_gate_shared_by_all_tokens_as_a_view(mp, dtype, n):
    """A tokens x n gate whose rows are one row (stride 0) has a gradient of its own for every token."""
    rng = np.random.default_rng(20)
    (R, _), (B, _), (WP, _), (G, _), (WQ, _) = norm_case(rng, 7, n, dtype, False, 0)
    DR, DY = matrix(rng, 7, n, dtype)[0], matrix(rng, 7, n, dtype)[0]
    shared = G[None].expand(7, n)
    assert shared.stride(0) == 0
    whole = shared.contiguous()
    for a, b in zip(mp.block_norm(R, B, WP, shared, WQ), mp.block_norm(R, B, WP, whole, WQ)):
        assert torch.equal(a, b)
    want = mp.block_norm_backward(DR, DY, R, B, WP, whole, WQ)
    got = mp.block_norm_backward(DR, DY, R, B, WP, shared, WQ)
    assert got[3].shape == (7, n) and got[3].dtype == TYPES[dtype]
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def gelu_tail_bounds(g, dtype):
    """Phi(g) for negative g and the relative error its computation may have.  16 bits: that of Abramowitz and Stegun 7.1.26 as a
    form of Phi(-|g|), here in 64 bits, the roundings of its terms and of the exponential's argument; fp32: those of erfc's
    argument, g^2 times over, and 16 of the function's."""
    from scipy import special
    phi, x = special.ndtr(g), np.abs(g) * np.sqrt(0.5)
    if dtype == "f32":
        return phi, (3 * g * g + 16) * U32
    c = np.array([0.254829592, -0.284496736, 1.421413741, -1.453152027, 1.061405429])
    t = 1 / (1 + 0.3275911 * x)
    terms = c[:, None] * t[None] ** np.arange(1, 6)[:, None]
    formula = 0.5 * terms.sum(0) * np.exp(-x * x)
    return phi, np.abs(formula / phi - 1) + (12 * np.abs(terms).sum(0) / terms.sum(0) + 3 * g * g + 16) * U32


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_gelu_keeps_its_digits_where_it_fades_out(mp, dtype):
    """One token per pre-activation g from -6 to 0, G = g and U = 2^13 exactly: gelu(g) and its slope to their own digits."""
    g = np.concatenate([-np.linspace(0.03, 6, 700), -np.arange(1, 24) / 4.0])
    g = torch.from_numpy(g).to(TYPES[dtype]).double().numpy()
    u = 2.0 ** 13
    X = torch.from_numpy(np.stack([g, np.ones_like(g)], 1)).to(TYPES[dtype]).cuda()
    Wg = torch.tensor([[1.0], [0.0]], dtype=TYPES[dtype], device="cuda")
    Wu = torch.tensor([[0.0], [u]], dtype=TYPES[dtype], device="cuda")
    phi, rel = gelu_tail_bounds(g, dtype)
    density = np.exp(-0.5 * g * g) / np.sqrt(2 * np.pi)
    H = g * phi * u
    close(mp.gated_ff(X, Wg, Wu, act="gelu"), H[:, None], (rel * np.abs(H) + 4 * U32 * np.abs(H) + stored(H, dtype))[:, None], "H")
    # dG = U slope is the first column of dX, rounded once more as an operand
    slope = phi + g * density
    dX = mp.gated_ff_backward(torch.ones(len(g), 1, dtype=TYPES[dtype], device="cuda"), X, Wg, Wu, act="gelu", need_dw=False)[0]
    e = u * (rel * phi + np.abs(g) * density * (3 * g * g + 16) * U32 + 4 * U32 * np.abs(slope))
    close(dX[:, 0], slope * u, e + 2.01 * stored(slope * u, dtype), "dG")


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_w4_pack_does_not_lose_a_nan(mp, dtype, group):
    """A group that holds a NaN (or an infinity, for which 4 bits have no code) makes its column's products NaN and no others."""
    rng = np.random.default_rng(21)
    W, _ = matrix(rng, 200, 40, dtype, 0.1)
    W[:, 7] = 0
    X, _ = matrix(rng, 3, 200, dtype)
    clean = mp.w4_matvec(X, mp.w4_pack(W, group))
    bad = W.clone()
    bad[130, 3], bad[0, 7], bad[199, 20], bad[50, 39] = float("nan"), float("nan"), float("inf"), float("-inf")
    got = mp.w4_matvec(X, mp.w4_pack(bad, group))
    off = torch.zeros(40, dtype=torch.bool, device="cuda")
    off[[3, 7, 20, 39]] = True
    assert torch.isnan(got[:, off]).all()
    assert torch.equal(got[:, ~off], clean[:, ~off])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [1, 5, 33])
def test_w4_products_of_infinite_tokens(mp, dtype, tokens):
    """An infinity in a token is one in its products, by the sign of the weight, and NaN where the weight is 0."""
    rng = np.random.default_rng(22)
    for n, m in ((100, 40), (700, 300)):
        W, w = w4_matrix(mp, rng, n, m, 64)
        X, x = matrix(rng, tokens, n, dtype)
        X[tokens // 2, 65] = x[tokens // 2, 65] = float("inf")
        with np.errstate(invalid="ignore"):
            want = x @ w
        got = values(mp.w4_matvec(X, W))
        row = tokens // 2
        assert np.isinf(want[row]).any() and np.isnan(want[row]).any()
        assert np.array_equal(got[row], want[row], equal_nan=True)
        rest = np.arange(tokens) != row
        assert np.isfinite(got[rest]).all()


@pytest.mark.parametrize("tokens", [5, 40, 300])
def test_gated_ff_fp32_infinities_are_the_definition_s(mp, tokens):
    """Infinities of either sign in tokens, weights and gradients come out as sums in fp32 have them, at any number of tokens: the
    signs of infinities and the places of NaN are those of the 64-bit form, and what they do not reach keeps its bits."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(23)
    new = lambda r, c, s=1.0: torch.randn(r, c, generator=gen, device="cuda") * s  # noqa: E731
    n, m, inf = 200, 333, float("inf")
    X, Wg, Wu, dH = new(tokens, n), new(n, m, 0.1), new(n, m, 0.1), new(tokens, m)
    X[3, 5], X[4, 100], X[4, 199], Wu[7, 40], Wg[7, 41] = inf, -inf, inf, -inf, inf
    G, U = torch.empty(2, tokens, m, device="cuda")
    H = mp.gated_ff(X, Wg, Wu, act="relu", g_out=G, u_out=U)
    for got, W in ((G, Wg), (U, Wu)):
        with np.errstate(invalid="ignore"):
            want = values(X) @ values(W)
        assert np.isinf(want[3]).all() and np.isinf(want[:3, 40 if W is Wu else 41]).all() and np.isnan(want[4]).any()
        special = ~np.isfinite(want)
        assert np.array_equal(values(got)[special], want[special], equal_nan=True)
        assert np.isfinite(values(got)[~special]).all()
    clean = mp.gated_ff(X.nan_to_num(0.5, 0.5, 0.5), Wg.nan_to_num(0.1, 0.1, 0.1), Wu.nan_to_num(0.1, 0.1, 0.1), act="relu")
    rows = [t for t in range(tokens) if t not in (3, 4)]
    cols = [c for c in range(m) if c not in (40, 41)]
    assert torch.equal(H[rows][:, cols], clean[rows][:, cols])
    # gradients: one infinity in dH, weights and tokens finite
    X, Wg, Wu = X.nan_to_num(0.5, 0.5, 0.5), Wg.nan_to_num(0.1, 0.1, 0.1), Wu.nan_to_num(0.1, 0.1, 0.1)
    dH[2, 50] = -inf
    got = mp.gated_ff_backward(dH, X, Wg, Wu, act="silu")
    with np.errstate(invalid="ignore"):
        want = bo.gated_ff_backward(values(dH), values(X), values(Wg), values(Wu), "silu")
    for t, w in zip(got, want):
        special = ~np.isfinite(w)
        assert special.any()
        assert np.array_equal(values(t)[special], w[special], equal_nan=True)
        assert np.isfinite(values(t)[~special]).all()


def test_gated_ff_without_tokens_of_more_entries_than_a_launch_has_threads(mp):
    """2^32 entries in each gradient."""
    n, m = 1 << 16, 1 << 16
    X, dH = torch.empty(0, n, dtype=torch.bfloat16, device="cuda"), torch.empty(0, m, dtype=torch.bfloat16, device="cuda")
    W = torch.empty(n, m, dtype=torch.bfloat16, device="cuda")
    dWg, dWu = torch.empty_like(W), torch.empty_like(W)
    for t in (dWg, dWu):
        t.view(torch.int16).fill_(0x4040)
    mp.gated_ff_backward(dH, X, W, W, dWg=dWg, dWu=dWu, need_dx=False)
    for t in (dWg, dWu):
        for rows in t.view(torch.int16).split(1 << 13):
            assert not rows.any()


@pytest.mark.parametrize("masked", [False, True])
def test_gated_ff_elementwise_passes_of_several_strides(mp, masked):
    """Slopes of 2^26 + entries and copies of 2^27 +: more than their grids have threads at a time."""
    tokens, n, m = 8200, 9, 8331
    gen = torch.Generator(device="cuda")
    gen.manual_seed(25)
    new = lambda r, c, s=1.0: (torch.randn(r, c, generator=gen, device="cuda") * s).to(torch.bfloat16)  # noqa: E731
    X, Wg, Wu, dH = new(tokens, n), new(n, m, 0.3), new(n, m, 0.3), new(tokens, m)
    mask = (torch.rand(m, generator=gen, device="cuda") < 0.5).to(torch.uint8) if masked else None
    want = exact_block(X, Wg, Wu, dH, "silu", mask)
    G, U = want["G"].to(torch.bfloat16), want["U"].to(torch.bfloat16)
    for name, t in zip(("dX", "dWg", "dWu"), mp.gated_ff_backward(dH, X, Wg, Wu, mask=mask, G=G, U=U)):
        blocks_close(t, want[name], 1.5 * ROUND["bf16"], name)
    tokens, n, m = 20, 16411, 8201
    X, Wg, Wu = new(tokens, n), new(n, m, 0.01), new(n, m, 0.01)
    got = mp.gated_ff(X, Wg, Wu, mask=mask[:m].contiguous() if masked else None)
    h = torch.nn.functional.silu(X.double() @ Wg.double()) * (X.double() @ Wu.double())
    blocks_close(got, h * mask[:m] if masked else h, ROUND["bf16"], "H")


def test_block_norm_backward_of_more_columns_than_a_launch_has_threads_for(mp):
    """One row of 2^27 + 40 entries: the kernel that finishes the column sums gives 32 threads to each."""
    n = (1 << 27) + 40
    gen = torch.Generator(device="cuda")
    gen.manual_seed(26)
    r, dy = (torch.randn(1, n, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    w = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    dx, _, _, _, dw = mp.block_norm_backward(None, dy, r, w_pre=w)
    rms = (r.float().square().double().mean() + 1e-6).sqrt()
    want = (dy.double() * r.double())[0] / rms
    # one term per sum: the root's error, of 2^27 terms summed by 512 threads and a tree, and the products'
    assert (dw.double() - want).abs().le(want.abs() * ((1 << 18) + 64) * U32).all()
    assert torch.isfinite(dx).all() and dw[-40:].any() and dw[:40].any()


# ---------------------------------------------------------------- every form of the 4-bit launches, rows by the hundreds

def grid_matrix(rng, n, m, group):
    """A matrix that 4 bits hold exactly: codes times a power of two per column and group, the largest code in every group."""
    codes = rng.integers(0, 16, (n, m))
    codes[::group] = 7
    scale = 2.0 ** rng.integers(-4, 0, (-(-n // group), m))
    return np.where(codes >= 8, -bo.E2M1[codes & 7], bo.E2M1[codes & 7]) * np.repeat(scale, group, axis=0)[:n]


# tokens, n, m: column blocks (an odd number of them) and tokens that reach the launches of one to four column blocks per workgroup
W4_FORMS = [(1, 300, 8209), (3, 300, 8209), (5, 300, 8209), (4, 700, 200), (9, 700, 200), (8, 257, 16417), (16, 257, 16417), (33, 300, 16417),
            (64, 300, 16417), (1, 130, 16417)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("case", range(len(W4_FORMS)))
def test_w4_every_form(mp, case, dtype):
    tokens, n, m = W4_FORMS[case]
    rng = np.random.default_rng(27 + case)
    for group in (32, 64, 128):
        wg, wu = grid_matrix(rng, n, m, group), grid_matrix(rng, n, m, group)
        Wg, Wu = (mp.w4_pack(torch.from_numpy(w.astype(np.float32)).cuda(), group) for w in (wg, wu))
        X, x = matrix(rng, tokens, n, dtype, n ** -0.5, gap=group % 3)
        c = sum_bound(n, dtype)
        g, u = x @ wg, x @ wu
        eg, eu = c * (np.abs(x) @ np.abs(wg)), c * (np.abs(x) @ np.abs(wu))
        pad = torch.full((tokens + 1, m + 5), 7.0, dtype=TYPES[dtype], device="cuda")
        mp.w4_matvec(X, Wg, y=pad[:tokens, :m])
        close(pad[:tokens, :m], g, eg + stored(g, dtype), "y")
        assert (pad[tokens:] == 7).all() and (pad[:, m:] == 7).all()
        h, a = bo.activation("silu", g) * u, np.abs(bo.activation("silu", g))
        eh = (SLOPE * eg + 16 * U32 * (a + np.abs(g))) * (np.abs(u) + eu) + a * eu
        pad.fill_(7.0)
        mp.w4_gated_matvec(X, Wg, Wu, h=pad[:tokens, :m])
        close(pad[:tokens, :m], h, eh + stored(h, dtype), "h")
        assert (pad[tokens:] == 7).all() and (pad[:, m:] == 7).all()


# more rows than are resident at once, for every number of threads that a row has
NORM_ROWS = [(8300, 40), (8250, 250), (2200, 500), (1100, 1500), (600, 2500), (600, 3003), (300, 5001), (300, 8200), (300, 16390)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("token_gate", [False, True])
@pytest.mark.parametrize("i", range(len(NORM_ROWS)))
def test_block_norm_of_many_rows(mp, i, token_gate, dtype):
    tokens, n = NORM_ROWS[i]
    rng = np.random.default_rng(500 + i)
    eps, scale = 1e-5, 0.6
    (X, x), (B, b), (WP, wp), (G, g), (WQ, wq) = norm_case(rng, tokens, n, dtype, token_gate, i % 2)
    r, y, er, ey = norm_forward_bounds(x, b, wp, g, wq, scale, eps, dtype)
    R, Y = mp.block_norm(X, B, WP, G, WQ, scale=scale, eps=eps)
    close(R, r, er + stored(r, dtype), "r")
    close(Y, y, ey + stored(y, dtype), "y")
    Xc, Bc = X.clone(), B.clone()
    mp.block_norm(Xc, Bc, WP, G, WQ, scale=scale, eps=eps, r=Xc, y=Bc)
    assert torch.equal(Xc, R) and torch.equal(Bc, Y)

    (DR, dr), (DY, dy) = matrix(rng, tokens, n, dtype, gap=i % 2), matrix(rng, tokens, n, dtype, gap=i % 2)
    dx, db, dwp, dg, dwq = bo.block_norm_backward(dr, dy, x, b, wp, g, wq, scale, eps)
    ws = mp.Workspace(mp.block_norm_workspace_bytes(tokens, n))
    ws.buf.fill_(255)
    got = mp.block_norm_backward(DR, DY, X, B, WP, G, WQ, scale=scale, eps=eps, workspace=ws)
    k, over = (n + 64) * U32, (tokens + 16) * U32
    sr, sb, e, f = bo.rms(x, eps), bo.rms(b, eps), np.abs(wq * dy), np.abs(scale * g * wp)
    mag = np.abs(dr) + e / sr + np.abs(x) / sr * (np.abs(x) / sr * e).mean(1, keepdims=True) / sr
    bh = np.abs(b) / sb
    close(got[0], dx, k * mag + stored(dx, dtype), "dx")
    close(got[1], db, 4 * k * (f * mag / sb + bh * (bh * f * mag).mean(1, keepdims=True) / sb) + stored(db, dtype), "db")
    close(got[2], dwp, (4 * k + over) * (np.abs(scale * g) * mag * bh).sum(0) + 1e-37, "dw_post")
    tg = np.abs(scale * wp) * mag * bh
    if token_gate:
        close(got[3], dg, 4 * k * tg + stored(dg, dtype), "dgate")
    else:
        close(got[3], dg, (4 * k + over) * tg.sum(0) + 1e-37, "dgate")
    close(got[4], dwq, (k + over) * np.abs(dy * (x / sr)).sum(0) + 1e-37, "dw_pre")
    # in place: dx over dr, db over b, then over dy
    DRc, Bc = DR.clone(), B.clone()
    for a, c in zip(got, mp.block_norm_backward(DRc, DY, X, Bc, WP, G, WQ, scale=scale, eps=eps, dx=DRc, db=Bc)):
        assert torch.equal(a, c)
    DYc = DY.clone()
    for a, c in zip(got, mp.block_norm_backward(DR, DYc, X, B, WP, G, WQ, scale=scale, eps=eps, db=DYc)):
        assert torch.equal(a, c)


@pytest.mark.parametrize("m", range(4088, 4098))
def test_packed_channels_of_every_remainder(mp, m):
    """Widths around two whole segments of columns, one to eight channels pruned ahead of a full last segment."""
    tokens, n, dtype = 1024, 1032, "bf16"
    assert mp.gated_ff_route(TYPES[dtype], 1, tokens, n, m)["packed"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(m)
    new = lambda r, c, s=1.0: (torch.randn(r, c, generator=gen, device="cuda") * s).to(TYPES[dtype])  # noqa: E731
    X, Wg, Wu, dH = new(tokens, n), new(n, m, n ** -0.5), new(n, m, n ** -0.5), new(tokens, m)
    ws = mp.Workspace(mp.gated_ff_workspace_bytes(tokens, n, m, TYPES[dtype], True))
    for pruned in range(1, 9):
        mask = torch.ones(m, dtype=torch.uint8, device="cuda")
        mask[torch.randperm(2000, generator=gen, device="cuda")[:pruned]] = 0
        ws.buf.fill_(255)
        want = exact_block(X, Wg, Wu, dH, "silu", mask)
        for name, t in zip(("dX", "dWg", "dWu"), mp.gated_ff_backward(dH, X, Wg, Wu, mask=mask, workspace=ws)):
            blocks_close(t, want[name], 1.5 * ROUND[dtype], name)
