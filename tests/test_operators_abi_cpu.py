"""Host-side checks of the 4-bit, dropout and router calls: sizes, and refusals before any HIP call."""
import math
import os

import numpy as np
import pytest

from paper_2404_15159_amd import binding as B

FAKE = 0x10000   # non-null, 16-byte aligned, never dereferenced on these paths


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2404_15159_amd import build
        build.build(verbose=False)
    return B.load()


def code(fn, *args):
    with pytest.raises(B.MixLoraError) as e:
        fn(*args, stream=1 << 20)
    return e.value.code


NULL, SHAPE, DTYPE, ALIGN, WORKSPACE = -1, -2, -3, -4, -5


def lin(T=5, d_in=64, d_out=128, r=8, s=2.0, dtype=B.BF16):
    return B.LinearDims(T, d_in, d_out, r, s, dtype)


def test_array_sizes():
    assert B.mixlora_q4_code_bytes(16, 128) == 1024 and B.mixlora_q4_code_bytes(8, 8) == 1024
    assert B.mixlora_q4_code_bytes(24, 136) == 4096
    assert [B.mixlora_q4_scale_bytes(24, 136, g) for g in (32, 64, 128)] == [4 * 16 * n * 2 for n in (4, 2, 1)]
    assert B.mixlora_q4_code_bytes(11008, 4096) == 11008 * 4096 // 2
    for bad in ((0, 8), (8, 0), (12, 8), (8, 12), (-8, 8)):
        assert B.mixlora_q4_code_bytes(*bad) == 0 and B.mixlora_q4_scale_bytes(*bad, 64) == 0
    assert B.mixlora_q4_scale_bytes(8, 8, 16) == 0 and B.mixlora_q4_scale_bytes(8, 8, 0) == 0
    assert B.mixlora_q4_code_bytes(2 ** 31 - 8, 2 ** 31 - 8) == 0   # more tiles than a launch holds


@pytest.mark.parametrize("back", [False, True])
def test_quantize_refusals(back):
    q = B.make_q4(FAKE, FAKE, 64)
    call = ((lambda W, dt, n, k, q4: code(B.mixlora_q4_dequantize, q4, n, k, False, W, dt)) if back else
            (lambda W, dt, n, k, q4: code(B.mixlora_q4_quantize, W, dt, n, k, q4)))
    assert call(None, B.BF16, 16, 128, q) == NULL
    assert call(FAKE, B.BF16, 16, 128, None) == NULL
    assert call(FAKE, B.BF16, 16, 128, B.make_q4(None, FAKE, 64)) == NULL
    assert call(FAKE, B.BF16, 16, 128, B.make_q4(FAKE, None, 64)) == NULL
    assert call(FAKE, 2, 16, 128, q) == DTYPE
    for n, k in ((12, 128), (16, 100), (0, 128), (16, -8)):
        assert call(FAKE, B.F32, n, k, q) == SHAPE
    assert call(FAKE, B.F32, 16, 128, B.make_q4(FAKE, FAKE, 48)) == SHAPE
    assert call(FAKE + 2, B.BF16, 16, 128, q) == ALIGN
    assert call(FAKE, B.BF16, 16, 128, B.make_q4(FAKE + 8, FAKE, 64)) == ALIGN
    assert call(FAKE, B.BF16, 16, 128, B.make_q4(FAKE, FAKE + 2, 64)) == ALIGN
    if back:
        assert code(B.mixlora_q4_dequantize, q, 16, 128, 2, FAKE, B.BF16) == SHAPE


def test_workspace_sizes():
    for fn in (lambda d, b: B.mixlora_q4_linear_workspace_bytes(d, 64, b), B.mixlora_lora_dropout_workspace_bytes):
        assert 0 < fn(lin(), False) <= fn(lin(), True)
        for bad in (lin(T=0), lin(T=1 << 24), lin(d_in=60), lin(d_out=4), lin(r=0), lin(r=65), lin(dtype=3),
                    lin(d_in=1 << 27), lin(d_out=1 << 27)):
            assert fn(bad, False) == 0 and fn(bad, True) == 0
    assert B.mixlora_q4_linear_workspace_bytes(lin(), 96, True) == 0
    # the largest the limits allow stay positive 64-bit numbers
    assert B.mixlora_q4_linear_workspace_bytes(lin(T=(1 << 24) - 1, d_in=1 << 17, d_out=1 << 17), 32, True) > 1 << 40


W, Q = FAKE, None


def linear_calls(kind):
    """forward and backward as functions of keyword changes"""
    def fwd(d=lin(), q=(FAKE, FAKE, 64), A=FAKE, Bm=FAKE, drop=None, x=FAKE, y=FAKE, ws=FAKE, n=1 << 40, **_):
        if kind == "q4":
            return code(B.mixlora_q4_linear_forward, d, B.make_q4(*q), A, Bm, drop, x, y, ws, n)
        return code(B.mixlora_lora_dropout_forward, d, q[0], A, Bm, drop, x, y, ws, n)

    def bwd(d=lin(), q=(FAKE, FAKE, 64), A=FAKE, Bm=FAKE, drop=None, x=FAKE, dy=FAKE, ws=FAKE, n=1 << 40, dx=FAKE,
            dA=FAKE, dB=FAKE, W_T=None, **_):
        if kind == "q4":
            return code(B.mixlora_q4_linear_backward, d, B.make_q4(*q), A, Bm, drop, x, dy, ws, n, dx, dA, dB)
        return code(B.mixlora_lora_dropout_backward, d, q[0], W_T, A, Bm, drop, x, dy, ws, n, dx, dA, dB)
    return fwd, bwd


@pytest.mark.parametrize("kind", ["q4", "dropout"])
def test_linear_refusals(kind):
    fwd, bwd = linear_calls(kind)
    for call, names in ((fwd, ("A", "Bm", "x", "y", "ws")), (bwd, ("A", "Bm", "x", "dy", "ws", "dx", "dA", "dB"))):
        for n in names:
            assert call(**{n: None}) == NULL, n
            assert call(**{n: FAKE + 4}) == ALIGN, n
        assert call(q=(None, FAKE, 64)) == NULL
        assert call(q=(FAKE + 4, FAKE, 64)) == ALIGN
        for bad in (lin(T=0), lin(T=1 << 24), lin(d_in=60), lin(d_out=4), lin(r=0), lin(r=65)):
            assert call(d=bad) == SHAPE
        assert call(d=lin(dtype=7)) == DTYPE
        for p in (-0.1, 1.0, 2.0, math.nan, math.inf, float(np.float32(1 - 2 ** -18))):
            assert call(drop=B.make_dropout(p, 1, 2)) == SHAPE, p
        assert call(drop=B.make_dropout(0.1, 1, 2, FAKE + 4)) == ALIGN
        size = (lambda b: B.mixlora_q4_linear_workspace_bytes(lin(), 64, b)) if kind == "q4" else \
            (lambda b: B.mixlora_lora_dropout_workspace_bytes(lin(), b))
        assert call(n=size(call is bwd) - 1) == WORKSPACE
        if kind == "q4":
            assert call(q=(FAKE, None, 64)) == NULL
            assert call(q=(FAKE, FAKE + 8, 64)) == ALIGN
            assert call(q=(FAKE, FAKE, 256)) == SHAPE
    if kind == "dropout":
        assert bwd(W_T=FAKE + 2) == ALIGN


def rd(T=10, N=8, k=2, mode=B.AUX_TOP1, dtype=B.F32):
    return B.RouterDims(T, N, k, 0.01, 0.001, mode, dtype)


def test_router_refusals():
    good = dict(d=rd(), logits=FAKE, mask=None, loss=FAKE, counts=FAKE, idx=FAKE, w=FAKE, ws=FAKE, n=1 << 30)

    def fwd(**kw):
        a = {**good, **kw}
        return code(B.mixlora_router_loss_forward, a["d"], a["logits"], a["mask"], a["loss"], a["counts"], a["idx"],
                    a["w"], a["ws"], a["n"])

    def bwd(d=rd(), logits=FAKE, idx=FAKE, dw=FAKE, ws=FAKE, n=1 << 30, out=FAKE):
        return code(B.mixlora_router_loss_backward, d, logits, None, idx, dw, 1.0, 1.0, ws, n, out)

    for n in ("logits", "loss", "counts", "idx", "w", "ws"):
        assert fwd(**{n: None}) == NULL and fwd(**{n: FAKE + 4}) == ALIGN, n
    for n in ("logits", "ws", "out", "idx"):
        assert bwd(**{n: None}) == NULL, n
    for n in ("logits", "ws", "out", "idx", "dw"):
        assert bwd(**{n: FAKE + 4}) == ALIGN, n
    for bad in (rd(T=0), rd(N=0), rd(N=65), rd(k=0), rd(k=9), rd(T=1 << 23)):
        assert fwd(d=bad) == SHAPE and bwd(d=bad) == SHAPE and B.mixlora_router_loss_workspace_bytes(bad) == 0
    for bad in (rd(mode=2), rd(dtype=4)):
        assert fwd(d=bad) == DTYPE and bwd(d=bad) == DTYPE
    need = B.mixlora_router_loss_workspace_bytes(rd())
    assert fwd(n=need - 1) == WORKSPACE and bwd(n=need - 1) == WORKSPACE
