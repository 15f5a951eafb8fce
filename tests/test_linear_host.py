"""Host-side checks of the product with an epilogue, dropout and the operators in 8 bits that need no GPU: sizes and refusals
before anything is enqueued."""
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


def drop(p=0.1, seed=1, offset=0, step=None):
    return ctypes.pointer(binding.DropoutStruct(p, seed, offset, step))


def block(tokens=4, n=8, m=16, X=P, ldx=8, W=P, ldw=16, bias=None, dropout=None):
    return binding.LinearBlock(tokens, n, m, X, ldx, W, ldw, bias, dropout)


def forward(lib, b, storage=1, act=0, residual=None, ldr=0, Y=P, ldy=16, Z=None, ldz=0, ws=P, nbytes=BIG):
    return lib.linear_forward(storage, act, None if b is None else ctypes.byref(b), residual, ldr, Y, ldy, Z, ldz, ws, nbytes, None)


def backward(lib, b, storage=1, act=0, dY=P, lddy=16, Z=P, ldz=16, dX=P, lddx=8, dW=P, lddw=16, dbias=P, ws=P, nbytes=BIG):
    return lib.linear_backward(storage, act, None if b is None else ctypes.byref(b), dY, lddy, Z, ldz, dX, lddx, dW, lddw, dbias, ws,
                               nbytes, None)


@pytest.mark.parametrize("call", [forward, backward])
def test_linear_refusals(lib, call):
    assert call(lib, None) == NULL
    assert call(lib, block(), storage=3) == VARIANT
    assert call(lib, block(), act=4) == VARIANT
    assert call(lib, block(), act=-1) == VARIANT
    for bad in (dict(tokens=-1), dict(n=0), dict(m=0), dict(ldx=7), dict(ldw=15)):
        assert call(lib, block(**bad)) == DIM, bad
    assert call(lib, block(n=1 << 31, ldx=1 << 31)) == LARGE
    assert call(lib, block(ldx=1 << 31)) == LARGE
    assert call(lib, block(n=1 << 20, m=1 << 20, ldx=1 << 20, ldw=1 << 20)) == LARGE
    for name in ("X", "W"):
        assert call(lib, block(**{name: None})) == NULL
        assert call(lib, block(**{name: P + 1})) == ALIGN
    for p in (-0.1, 1.0, 1.5, float("nan"), float("inf")):
        assert call(lib, block(dropout=drop(p))) == VALUE, p
    assert call(lib, block(dropout=drop(step=P + 4))) == ALIGN
    assert call(lib, block(), ws=None) == NULL
    assert call(lib, block(), ws=P + 64) == WS
    assert call(lib, block(), nbytes=16) == WS


def test_linear_refusals_of_one_direction(lib):
    assert forward(lib, block(bias=P + 1)) == ALIGN
    assert forward(lib, block(), residual=P, ldr=15) == DIM
    assert forward(lib, block(), residual=P + 1, ldr=16) == ALIGN
    assert forward(lib, block(), Y=None) == NULL
    assert forward(lib, block(), ldy=15) == DIM
    assert forward(lib, block(), Z=P, ldz=15) == DIM
    assert backward(lib, block(), dY=None) == NULL
    assert backward(lib, block(), lddy=15) == DIM
    assert backward(lib, block(), Z=None) == NULL
    assert backward(lib, block(), lddx=7) == DIM
    assert backward(lib, block(), lddw=15) == DIM
    assert backward(lib, block(), dX=P + 1) == ALIGN
    assert backward(lib, block(), dbias=P + 2) == ALIGN
    # no tokens: nothing to read, nothing to write
    assert forward(lib, block(tokens=0, X=None, W=None), Y=None) == OK


def test_gated_blocks_have_an_activation(lib):
    gated = binding.GatedBlock(4, 8, 16, P, 8, P, P, 16, None)
    assert lib.gated_ff_forward(1, binding.ACT_NONE, ctypes.byref(gated), P, 16, None, None, 0, P, BIG, None) == VARIANT


def test_linear_workspace(lib):
    out = ctypes.c_size_t(0)
    ask = lib.mlproj_linear_workspace_bytes
    assert ask(1, 4, 8, 16, 0, None) == NULL
    assert ask(3, 4, 8, 16, 0, ctypes.byref(out)) == VARIANT
    assert ask(1, 4, 0, 16, 0, ctypes.byref(out)) == DIM
    assert ask(1, 4, 8, 16, 2, ctypes.byref(out)) == DIM
    assert ask(1, 1 << 20, 1 << 20, 16, 0, ctypes.byref(out)) == LARGE
    for storage in (0, 1, 2):
        for tokens, n, m in ((0, 3, 5), (1, 1, 1), (1, 16384, 4096), (777, 2731, 1001), (4096, 16384, 4096), (300, 64, 8192)):
            for back in (0, 1):
                assert ask(storage, tokens, n, m, back, ctypes.byref(out)) == OK
                assert 0 < out.value < 16 << 30


def test_dropout_refusals(lib):
    def call(d, storage=1, tokens=4, n=8, x=P, ldx=8, residual=None, ldr=0, y=P, ldy=8):
        return lib.dropout_forward(storage, d, tokens, n, x, ldx, residual, ldr, y, ldy, None)
    assert call(None) == NULL
    assert call(drop(), storage=3) == VARIANT
    assert call(drop(), tokens=-1) == DIM
    assert call(drop(), n=0) == DIM
    assert call(drop(), tokens=1 << 20, n=1 << 20, ldx=1 << 20, ldy=1 << 20) == LARGE
    assert call(drop(), n=1 << 31, ldx=1 << 31, ldy=1 << 31) == LARGE
    for p in (-1e-9, 1.0, float("nan")):
        assert call(drop(p)) == VALUE
    assert call(drop(step=P + 1)) == ALIGN
    assert call(drop(), x=None) == NULL
    assert call(drop(), y=None) == NULL
    assert call(drop(), ldx=7) == DIM
    assert call(drop(), ldy=7) == DIM
    assert call(drop(), residual=P, ldr=7) == DIM
    assert call(drop(), residual=P + 1, ldr=8) == ALIGN
    assert call(drop(), tokens=0, x=None, y=None) == OK


def q8(rows=4, n=200, codes=P, ld=256, scales=P, lds=8):
    return binding.PackedQ8(rows, n, codes, ld, scales, lds)


BAD_Q8 = [(dict(codes=None), NULL), (dict(scales=None), NULL), (dict(ld=255), DIM), (dict(lds=7), DIM), (dict(ld=264), ALIGN), (dict(lds=9), ALIGN),
          (dict(codes=P + 8), ALIGN), (dict(scales=P + 2), ALIGN), (dict(ld=1 << 31), LARGE), (dict(lds=1 << 31), LARGE)]


def test_q8_pack_refusals(lib):
    def call(q, storage=1, by_columns=0, A=P, lda=200):
        return lib.q8_pack(storage, by_columns, A, lda, None if q is None else ctypes.byref(q), None)
    assert call(None) == NULL
    assert call(q8(), storage=3) == VARIANT
    assert call(q8(), by_columns=2) == VARIANT
    assert call(q8(rows=-1)) == DIM
    assert call(q8(n=0)) == DIM
    assert call(q8(rows=1 << 20, n=1 << 20)) == LARGE
    for bad, status in BAD_Q8:
        assert call(q8(**bad)) == status, bad
    assert call(q8(), A=None) == NULL
    assert call(q8(), A=P + 1) == ALIGN
    assert call(q8(), lda=199) == DIM
    assert call(q8(), by_columns=1, lda=3) == DIM
    assert call(q8(rows=0, codes=None, scales=None), A=None) == OK


def test_block_norm8_refusals(lib):
    def norm(tokens=4, n=200, b=P, ldb=200, w_post=P, gate=P, gate_stride=0, w_pre=P, scale=1.0, eps=1e-6):
        return binding.NormBlock(tokens, n, b, ldb, w_post, gate, gate_stride, w_pre, scale, eps)

    def call(k, y, storage=1, x=P, ldx=200, r=P, ldr=200):
        return lib.block_norm8_forward(storage, None if k is None else ctypes.byref(k), x, ldx, r, ldr, None if y is None else ctypes.byref(y), None)
    assert call(None, q8()) == NULL
    assert call(norm(), None) == NULL
    assert call(norm(w_pre=None), q8()) == NULL
    assert call(norm(), q8(), storage=3) == VARIANT
    assert call(norm(n=0), q8()) == DIM
    assert call(norm(), q8(n=201)) == DIM
    assert call(norm(), q8(rows=5)) == DIM
    assert call(norm(eps=-1.0), q8()) == VALUE
    assert call(norm(), q8(), x=None) == NULL
    assert call(norm(), q8(), r=None) == NULL
    assert call(norm(), q8(), ldx=199) == DIM
    assert call(norm(b=None), q8()) == NULL
    for bad, status in BAD_Q8:
        assert call(norm(), q8(**bad)) == status, bad
    assert call(norm(tokens=0, b=None, gate=None), q8(rows=0, codes=None, scales=None), x=None, r=None) == OK


def test_q8_product_refusals(lib):
    def linear(x, W, storage=1, act=3, bias=None, residual=None, ldr=0, y=P, ldy=16, ws=P, nbytes=BIG):
        return lib.q8_linear(storage, act, None if x is None else ctypes.byref(x), None if W is None else ctypes.byref(W), bias, residual, ldr, y,
                             ldy, ws, nbytes, None)

    def gated(x, W, storage=1, act=0, Wu=None, h=P, ldh=16, ws=P, nbytes=BIG):
        Wu = Wu or W
        return lib.q8_gated(storage, act, None if x is None else ctypes.byref(x), None if W is None else ctypes.byref(W),
                            None if Wu is None else ctypes.byref(Wu), h, ldh, ws, nbytes, None)
    x, W = q8(), q8(rows=16)
    for call in (linear, gated):
        assert call(None, W) == NULL
        assert call(x, None) == NULL
        assert call(x, W, storage=3) == VARIANT
        assert call(x, W, act=-1) == VARIANT
        assert call(x, q8(rows=16, n=201)) == DIM
        assert call(q8(rows=-1), W) == DIM
        assert call(q8(rows=1 << 31), W) == LARGE
        assert call(q8(rows=1 << 20), q8(rows=1 << 20)) == LARGE
        for bad, status in BAD_Q8:
            assert call(q8(**bad), W) == status, bad
            assert call(x, q8(rows=16, **bad)) == status, bad
        # rows of a tile are reached by 32-bit offsets
        assert call(q8(ld=(1 << 22) + 16), W) == LARGE
        assert call(x, W, ws=None) == NULL
        assert call(x, W, ws=P + 16) == WS
        assert call(x, W, nbytes=8) == WS
        assert call(q8(rows=0, codes=None, scales=None), q8(rows=16, codes=None, scales=None)) == OK
    assert linear(x, W, act=4) == VARIANT
    assert gated(x, W, act=3) == VARIANT
    assert linear(x, W, y=None) == NULL
    assert linear(x, W, ldy=15) == DIM
    assert linear(x, W, bias=P + 1) == ALIGN
    assert linear(x, W, residual=P, ldr=15) == DIM
    assert gated(x, W, h=None) == NULL
    assert gated(x, W, ldh=15) == DIM
    assert gated(x, W, Wu=q8(rows=17)) == DIM
    assert gated(x, W, Wu=q8(rows=16, ld=384)) == DIM
    assert gated(x, W, Wu=q8(rows=16, lds=12)) == DIM


def test_q8_workspace(lib):
    out = ctypes.c_size_t(0)
    ask = lib.mlproj_q8_workspace_bytes
    assert ask(4, 8, 16, 0, None) == NULL
    assert ask(4, 0, 16, 0, ctypes.byref(out)) == DIM
    assert ask(4, 8, 16, 2, ctypes.byref(out)) == DIM
    assert ask(1 << 20, 1 << 20, 16, 0, ctypes.byref(out)) == LARGE
    # more columns than a launch has threads for
    assert ask(1, 1, 1 << 30, 0, ctypes.byref(out)) == LARGE
    for sizes in ((0, 3, 5), (1, 1, 1), (1, 4096, 16384), (4096, 16384, 4096), (300, 64, 8192)):
        for gated in (0, 1):
            assert ask(*sizes, gated, ctypes.byref(out)) == OK
            assert 0 < out.value < 16 << 30


def test_dropout_object_is_fixed():
    """Its mask is its own: a program that advances an attribute would get the old mask again."""
    d = binding.Dropout(0.1, 3, 7)
    for name, value in (("p", 0.2), ("seed", 4), ("offset", 8), ("step", None)):
        with pytest.raises(AttributeError):
            setattr(d, name, value)
    assert (d.p, d.seed, d.offset, d.step) == (0.1, 3, 7, None)
    assert (d._struct.p, d._struct.seed, d._struct.offset) == (0.1, 3, 7)


def test_a_workspace_is_that_of_a_call_s_own_sizes(lib):
    """Fewer tokens may need more: their sums are cut into shares.  Less than the size of the call is refused."""
    out = ctypes.c_size_t(0)

    def linear(storage, tokens, back):
        assert lib.mlproj_linear_workspace_bytes(storage, tokens, 16384, 4096, back, ctypes.byref(out)) == OK
        return out.value

    def eight(tokens):
        assert lib.mlproj_q8_workspace_bytes(tokens, 16384, 4096, 0, ctypes.byref(out)) == OK
        return out.value
    assert linear(0, 300, 0) > linear(0, 4096, 0) and linear(1, 512, 1) > linear(1, 1024, 1) and eight(300) > eight(4096)
    for tokens in (300, 4096):
        b = block(tokens, 16384, 4096, ldx=16384, ldw=4096)
        assert forward(lib, b, storage=0, ldy=4096, nbytes=linear(0, tokens, 0) - 1) == WS
        assert backward(lib, b, lddy=4096, ldz=4096, lddx=16384, lddw=4096, nbytes=linear(1, tokens, 1) - 1) == WS
        x, W = q8(tokens, 16384, ld=16384, lds=512), q8(4096, 16384, ld=16384, lds=512)
        assert lib.q8_linear(1, 3, ctypes.byref(x), ctypes.byref(W), None, None, 0, P, 4096, P, eight(tokens) - 1, None) == WS
    # (a call without tokens enqueues nothing)
    assert forward(lib, block(0, 16384, 4096, X=None, ldx=16384, W=None, ldw=4096), storage=0, Y=None, nbytes=linear(0, 0, 0)) == OK
