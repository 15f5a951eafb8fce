"""Host-side checks of the pruned feed-forward block that need no GPU: sizes, routes, refusals before anything is enqueued."""
import ctypes
import os

import pytest

from paper_2405_02086_amd import binding

P = 1 << 20                 # non-null, 256-aligned; never dereferenced on these paths
BIG = 1 << 40
OK, NULL, DIM, LARGE, WS, VARIANT, ALIGN, VALUE = 0, -1, -2, -3, -5, -6, -7, -10


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        binding.build()
    return binding.lib()


def block(tokens=4, n=8, m=16, X=P, ldx=8, Wg=P, Wu=P, ldw=16, mask=None):
    return binding.GatedBlock(tokens, n, m, X, ldx, Wg, Wu, ldw, mask)


def forward(lib, b, storage=1, act=0, H=P, ldh=16, G=None, U=None, ldg=0, ws=P, nbytes=BIG):
    return lib.gated_ff_forward(storage, act, None if b is None else ctypes.byref(b), H, ldh, G, U, ldg, ws, nbytes, None)


def backward(lib, b, storage=1, act=0, dH=P, ldh=16, G=None, U=None, ldg=0, dX=P, lddx=8, dWg=P, dWu=P, lddw=16, ws=P, nbytes=BIG):
    return lib.gated_ff_backward(storage, act, None if b is None else ctypes.byref(b), dH, ldh, G, U, ldg, dX, lddx, dWg, dWu, lddw,
                                 ws, nbytes, None)


def test_status_of_a_bad_value(lib):
    assert lib.mlproj_status_string(VALUE) != b"unknown status"


@pytest.mark.parametrize("call", [forward, backward])
def test_gated_ff_refusals(lib, call):
    assert call(lib, None) == NULL
    assert call(lib, block(), storage=3) == VARIANT
    assert call(lib, block(), act=3) == VARIANT
    assert call(lib, block(), act=-1) == VARIANT
    for bad in (dict(tokens=-1), dict(n=0), dict(m=0), dict(ldx=7), dict(ldw=15)):
        assert call(lib, block(**bad)) == DIM, bad
    assert call(lib, block(n=1 << 31, ldx=1 << 31)) == LARGE
    assert call(lib, block(n=1 << 20, m=1 << 20, ldx=1 << 20, ldw=1 << 20)) == LARGE
    for name in ("X", "Wg", "Wu"):
        assert call(lib, block(**{name: None})) == NULL
        assert call(lib, block(**{name: P + 1})) == ALIGN
    assert call(lib, block(), ws=None) == NULL
    assert call(lib, block(), ws=P + 64) == WS
    assert call(lib, block(), nbytes=16) == WS
    assert call(lib, block(), G=P, ldg=16) == NULL
    assert call(lib, block(), U=P, ldg=16) == NULL
    assert call(lib, block(), G=P, U=P, ldg=15) == DIM
    assert call(lib, block(), G=P + 1, U=P, ldg=16) == ALIGN
    assert call(lib, block(), ldh=15) == DIM


def test_gated_ff_refusals_of_one_direction(lib):
    assert forward(lib, block(), H=None) == NULL
    assert forward(lib, block(), H=P + 1) == ALIGN
    assert backward(lib, block(), dH=None) == NULL
    assert backward(lib, block(), lddx=7) == DIM
    assert backward(lib, block(), lddw=15) == DIM
    assert backward(lib, block(), dWg=None) == NULL
    assert backward(lib, block(), dWu=None) == NULL
    assert backward(lib, block(), dX=P + 1) == ALIGN
    # no tokens: nothing to read, nothing to write
    assert forward(lib, block(tokens=0, X=None, Wg=None, Wu=None), H=None) == OK


def test_gated_ff_workspace(lib):
    out = ctypes.c_size_t(0)
    ask = lib.mlproj_gated_ff_workspace_bytes
    assert ask(1, 4, 8, 16, 0, 0, None) == NULL
    assert ask(3, 4, 8, 16, 0, 0, ctypes.byref(out)) == VARIANT
    assert ask(1, 4, 0, 16, 0, 0, ctypes.byref(out)) == DIM
    assert ask(1, 4, 8, 16, 2, 0, ctypes.byref(out)) == DIM
    assert ask(1, 4, 8, 16, 0, 2, ctypes.byref(out)) == DIM
    assert ask(1, 1 << 20, 1 << 20, 16, 0, 0, ctypes.byref(out)) == LARGE
    for storage in (0, 1, 2):
        for tokens, n, m in ((0, 3, 5), (1, 1, 1), (1, 4096, 16384), (777, 1001, 2731), (4096, 4096, 16384), (300, 8192, 64)):
            for back in (0, 1):
                sizes = []
                for masked in (0, 1):
                    assert ask(storage, tokens, n, m, back, masked, ctypes.byref(out)) == OK
                    sizes.append(out.value)
                assert 0 < sizes[0] <= sizes[1], "a workspace for masked calls serves the others"
                assert sizes[1] < 64 << 30


def test_gated_ff_routes(lib):
    """The rules' two sides: tiles by size, shares where rows are few, packing where products are long."""
    route = lambda storage, product, *dims: lib.mlproj_gated_ff_route(storage, product, *dims)  # noqa: E731
    assert route(1, 4, 4, 8, 16) == VARIANT
    assert route(7, 0, 4, 8, 16) == VARIANT
    assert route(1, 0, 4, 8, 0) == DIM
    kind = lambda r: r & 15       # noqa: E731
    shares = lambda r: r >> 8     # noqa: E731
    packed = lambda r: bool(r & 16)   # noqa: E731
    low = lambda r: bool(r & 64)      # noqa: E731
    for storage in (1, 2):
        big = route(storage, 0, 4096, 4096, 16384)
        assert kind(big) == 0 and not low(big) and shares(big) == 1 and packed(big)
        small = route(storage, 0, 16, 256, 128)
        assert kind(small) == 1 and low(small) and shares(small) == 1 and not packed(small)
        assert shares(route(storage, 0, 11, 7448, 1256)) > 1
        assert shares(route(storage, 2, 1000, 1000, 10000)) > 1
    assert kind(route(0, 0, 32, 256, 128)) == 3 and kind(route(0, 0, 33, 256, 128)) == 2
    assert kind(route(0, 2, 16, 256, 128)) == 2


def norm(tokens=4, n=8, b=P, ldb=8, w_post=P, gate=P, gate_stride=0, w_pre=P, scale=1.0, eps=1e-6):
    return binding.NormBlock(tokens, n, b, ldb, w_post, gate, gate_stride, w_pre, scale, eps)


def norm_forward(lib, k, storage=1, x=P, ldx=8, r=P, ldr=8, y=P, ldy=8):
    return lib.block_norm_forward(storage, None if k is None else ctypes.byref(k), x, ldx, r, ldr, y, ldy, None)


def norm_backward(lib, k, storage=1, r=P, ldr=8, dr=P, lddr=8, dy=P, lddy=8, dx=P, lddx=8, db=P, lddb=8, dw_post=P, dgate=P, ldg=0, dw_pre=P,
                  ws=P, nbytes=BIG):
    return lib.block_norm_backward(storage, None if k is None else ctypes.byref(k), r, ldr, dr, lddr, dy, lddy, dx, lddx, db, lddb,
                                   dw_post, dgate, ldg, dw_pre, ws, nbytes, None)


@pytest.mark.parametrize("call", [norm_forward, norm_backward])
def test_block_norm_refusals(lib, call):
    assert call(lib, None) == NULL
    assert call(lib, norm(), storage=-1) == VARIANT
    for bad in (dict(tokens=-1), dict(n=0), dict(ldb=7), dict(gate_stride=7)):
        assert call(lib, norm(**bad)) == DIM, bad
    assert call(lib, norm(n=1 << 31)) == LARGE
    for bad in (dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")), dict(scale=float("nan")), dict(scale=float("-inf"))):
        assert call(lib, norm(**bad)) == VALUE, bad
    assert call(lib, norm(b=None)) == NULL
    assert call(lib, norm(gate=None)) == NULL
    for name in ("b", "w_post", "gate", "w_pre"):
        assert call(lib, norm(**{name: P + 1})) == ALIGN


def test_block_norm_refusals_of_one_direction(lib):
    assert norm_forward(lib, norm(), x=None) == NULL
    assert norm_forward(lib, norm(), r=None) == NULL
    assert norm_forward(lib, norm(), y=None) == NULL
    assert norm_forward(lib, norm(), ldy=7) == DIM
    assert norm_backward(lib, norm(), r=None) == NULL
    assert norm_backward(lib, norm(), dy=None) == NULL
    assert norm_backward(lib, norm(), dx=None) == NULL
    assert norm_backward(lib, norm(), lddb=7) == DIM
    assert norm_backward(lib, norm(gate_stride=8), ldg=7) == DIM
    assert norm_backward(lib, norm(), dw_pre=P + 2) == ALIGN
    assert norm_backward(lib, norm(), ws=None) == NULL
    assert norm_backward(lib, norm(), nbytes=8) == WS
    assert norm_backward(lib, norm(), ws=P + 8) == WS
    out = ctypes.c_size_t(0)
    assert lib.mlproj_block_norm_workspace_bytes(4, 8, None) == NULL
    assert lib.mlproj_block_norm_workspace_bytes(4, 0, ctypes.byref(out)) == DIM
    assert lib.mlproj_block_norm_workspace_bytes(1 << 20, 8192, ctypes.byref(out)) == OK and out.value < 64 << 20
    assert norm_forward(lib, norm(tokens=0, b=None), x=None, r=None, y=None) == OK


def packed(n=100, m=40, group=64, codes=P, scales=P):
    return binding.PackedW4(n, m, group, codes, scales)


def test_w4_refusals(lib):
    a, b = ctypes.c_size_t(0), ctypes.c_size_t(0)
    assert lib.mlproj_w4_bytes(100, 40, 64, ctypes.byref(a), ctypes.byref(b)) == OK
    assert (a.value, b.value) == (3 * 1 * 1024, 3 * 1 * 16 * 2 * 2)
    assert lib.mlproj_w4_bytes(100, 40, 16, ctypes.byref(a), ctypes.byref(b)) == VARIANT
    assert lib.mlproj_w4_bytes(0, 40, 32, ctypes.byref(a), ctypes.byref(b)) == DIM
    assert lib.mlproj_w4_bytes(100, 40, 64, None, ctypes.byref(b)) == NULL
    R = ctypes.byref
    ok = packed()
    assert lib.w4_pack(5, P, 40, R(ok), None) == VARIANT
    assert lib.w4_pack(1, None, 40, R(ok), None) == NULL
    assert lib.w4_pack(1, P, 39, R(ok), None) == DIM
    assert lib.w4_pack(1, P + 1, 40, R(ok), None) == ALIGN
    assert lib.w4_pack(1, P, 40, R(packed(codes=None)), None) == NULL
    assert lib.w4_pack(1, P, 40, R(packed(codes=P + 8)), None) == ALIGN
    assert lib.w4_matvec(1, None, P, 100, 2, P, 40, None) == NULL
    assert lib.w4_matvec(1, R(packed(group=48)), P, 100, 2, P, 40, None) == VARIANT
    assert lib.w4_matvec(1, R(ok), None, 100, 2, P, 40, None) == NULL
    assert lib.w4_matvec(1, R(ok), P, 99, 2, P, 40, None) == DIM
    assert lib.w4_matvec(1, R(ok), P, 100, 2, P, 39, None) == DIM
    assert lib.w4_matvec(1, R(ok), P, 100, -1, P, 40, None) == DIM
    assert lib.w4_matvec(1, R(packed(scales=P + 2)), P, 100, 2, P, 40, None) == ALIGN
    assert lib.w4_matvec(1, R(packed(codes=None, scales=None)), None, 100, 0, None, 40, None) == OK
    assert lib.w4_gated_matvec(1, 0, R(ok), None, P, 100, 2, P, 40, None) == NULL
    assert lib.w4_gated_matvec(1, 3, R(ok), R(ok), P, 100, 2, P, 40, None) == VARIANT
    assert lib.w4_gated_matvec(1, 0, R(ok), R(packed(m=41)), P, 100, 2, P, 48, None) == DIM
    assert lib.w4_gated_matvec(1, 0, R(ok), R(packed(group=32)), P, 100, 2, P, 48, None) == DIM


def test_what_a_call_allocates_belongs_to_its_stream(monkeypatch):
    """Scratch is given back when a call returns, before its kernels ran: it has to come from the call's stream."""
    import contextlib
    import types
    import torch
    current, seen = ["default"], []

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    def empty(*args, **kw):
        seen.append(current[-1])
        return types.SimpleNamespace(data_ptr=lambda: 256)

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch, "empty_like", empty)
    like = types.SimpleNamespace(shape=(2, 3), is_contiguous=lambda: True, new_empty=empty)
    binding._import_torch()
    binding.Workspace(1000)
    binding.Workspace(1000, stream="side")
    binding._result(None, (2, 3), like, "same", None)
    binding._result(None, (2, 3), like, "same", "side")
    binding._result(None, (2, 4), like, "other", None)
    binding._result(None, (2, 4), like, "other", "side")
    assert seen == ["default", "side"] * 3


def test_gated_ff_sizes_past_one_launch_are_too_large(lib):
    """Products whose tiles would be 2^32 threads or more are refused as sizes, not at their launch."""
    out = ctypes.c_size_t(0)
    ask = lib.mlproj_gated_ff_workspace_bytes
    top = 1 << 30
    for storage in (0, 1, 2):
        assert ask(storage, 1, 1, top, 0, 0, ctypes.byref(out)) == LARGE
        assert ask(storage, 1, 1, top, 1, 1, ctypes.byref(out)) == LARGE
        assert ask(storage, 1, 1, top >> 3, 0, 0, ctypes.byref(out)) == OK
        assert ask(storage, 0, 1 << 16, 1 << 17, 1, 0, ctypes.byref(out)) == OK
        assert ask(storage, 0, 1, top, 1, 1, ctypes.byref(out)) == OK
        assert ask(storage, 1 << 18, 64, 1 << 16, 1, 1, ctypes.byref(out)) == OK
    big = block(tokens=1, n=1, m=top, ldx=1, ldw=top)
    assert forward(lib, big, ldh=top) == LARGE
    assert backward(lib, big, ldh=top, lddx=1, lddw=top) == LARGE
    assert forward(lib, block(tokens=32, n=1, m=1 << 28, ldx=1, ldw=1 << 28), storage=0, ldh=1 << 28) == LARGE


def test_block_norm_sizes_past_one_launch_are_too_large(lib):
    """2^23 rows of more than 2^14 entries would be 2^32 threads."""
    for tokens, n in ((1 << 23, 16385), (1 << 30, 129)):
        k = norm(tokens=tokens, n=n, ldb=n)
        assert norm_forward(lib, k, ldx=n, ldr=n, ldy=n) == LARGE
        assert norm_backward(lib, k, ldr=n, lddr=n, lddy=n, lddx=n, lddb=n) == LARGE


def test_w4_sizes_past_one_launch_are_too_large(lib):
    R = ctypes.byref
    wide, wider, widest = packed(m=1 << 28), packed(m=1 << 29), packed(m=1 << 30)
    for tokens, w in ((1, wide), (7, wide), (8, wider), (64, widest)):
        assert lib.w4_matvec(1, R(w), P, 100, tokens, P, w.m, None) == LARGE
        assert lib.w4_gated_matvec(1, 0, R(w), R(w), P, 100, tokens, P, w.m, None) == LARGE
    assert lib.w4_pack(1, P, 1 << 30, R(packed(m=1 << 30, group=32)), None) == LARGE
    assert lib.w4_matvec(1, R(wide), None, 100, 0, None, 1 << 28, None) == OK
