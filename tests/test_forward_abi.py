"""Refusals and workspace sizes of the forward-pass operators through the C ABI, without a device: arguments are checked before anything is
launched, so made-up addresses are enough."""
import ctypes

import numpy as np
import pytest

import forward_ref as ref
from paper_2601_12917_b200 import zgr

A = 0x10000      # never dereferenced on the host


def drop(x=A, ldx=16, bias=None, r=None, ldr=0, y=A, ldy=16, rows=4, cols=16, dtype=zgr.F32, p=0.1):
    return zgr.lib().zgr_dropout(x, ldx, bias, r, ldr, y, ldy, rows, cols, dtype, p, 1, 0, None)


@pytest.mark.parametrize("kw", [dict(x=None), dict(y=None), dict(ldx=15), dict(ldy=8), dict(r=A, ldr=3), dict(x=A + 2), dict(y=A + 1), dict(bias=A + 2), dict(r=A + 2, ldr=16),
                                dict(dtype=3), dict(dtype=-1), dict(p=-1e-9), dict(p=1.0001), dict(p=float("nan")), dict(rows=-1), dict(cols=-1), dict(ldx=-16),
                                dict(dtype=zgr.F16, x=A + 1), dict(ldx=1 << 62)])
def test_dropout_refuses(kw):
    assert drop(**kw) == zgr.EINVAL


def test_nothing_to_do_is_not_an_error():
    assert drop(rows=0) == zgr.OK and drop(cols=0, x=None, y=None) == zgr.OK
    L = zgr.lib()
    assert L.zgr_quantize_rows(None, 0, 0, 8, zgr.F32, None, 8, None, None) == zgr.OK
    assert L.zgr_linear_i8(None, 0, None, 0, None, None, None, 0, None, 0, 0, 5, 7, zgr.F32, 0.0, 0, 0, None, 0, None) == zgr.OK


def back(dy=A, dx=A, db=A, rows=10000, cols=64, ws=A, ws_bytes=None, dtype=zgr.F32, p=0.1):
    L = zgr.lib()
    need = L.zgr_dropout_backward_workspace(rows, cols)
    return L.zgr_dropout_backward(dy, cols, dx, cols, db, rows, cols, dtype, p, 1, 0, ws, need if ws_bytes is None else need + ws_bytes, None)


@pytest.mark.parametrize("kw", [dict(dy=None), dict(dx=None), dict(ws=None), dict(ws=A + 8), dict(ws_bytes=-1), dict(db=A + 2), dict(dtype=7), dict(p=2.0), dict(rows=-1)])
def test_dropout_backward_refuses(kw):
    assert back(**kw) == zgr.EINVAL


def test_sizes_whose_sums_would_pass_63_bits_are_refused():
    L, huge = zgr.lib(), (1 << 63) - 1
    assert drop(rows=1, cols=huge, ldx=0, ldy=0) == zgr.EINVAL and drop(rows=huge, cols=1, ldx=1, ldy=1) == zgr.EINVAL
    for rows, cols in ((1, huge), (huge, 1), (huge, huge)):
        assert L.zgr_dropout_backward_workspace(rows, cols) == zgr.EINVAL
        assert L.zgr_dropout_backward(A, cols, A, cols, A, rows, cols, zgr.F32, 0.5, 1, 0, A, huge, None) == zgr.EINVAL
    assert L.zgr_dropout_backward(A, 0, A, 0, A, 0, huge, zgr.F32, 0.5, 1, 0, A, huge, None) == zgr.EINVAL
    assert L.zgr_quantize_rows(A, 0, 1, huge, zgr.F32, A, 0, A, None) == zgr.EINVAL


def test_workspaces_cover_what_the_sizes_need():
    L = zgr.lib()
    for rows, cols in ((4096, 1024), (1 << 20, 8), (100000, 300), (129, 1000), (4097, 1)):
        b = L.zgr_dropout_backward_workspace(rows, cols)
        assert b % (4 * cols) == 0 and 2 <= b // (4 * cols) <= 592           # up to four ranges for each of 148 multiprocessors
    for rows, cols in ((1, 1), (1, 100000), (7, 5), (128, 1000), (4096, 1), (200, 128)):
        assert L.zgr_dropout_backward_workspace(rows, cols) == 0             # one range: its sums are the result
    assert L.zgr_dropout_backward_workspace(0, 8) == 0 and L.zgr_dropout_backward_workspace(-1, 8) == zgr.EINVAL
    for m, n, k in ((1, 11008, 4096), (2, 50265, 4096), (4, 2048, 4096), (8, 1024, 4096), (0, 8, 8)):      # quantised by the product itself
        assert L.zgr_linear_i8_workspace(m, n, k) == 0
    for m, n, k in ((9, 8, 16), (4, 8193, 16), (4, 4096, 4096), (8, 1025, 4096), (100, 50, 17), (8192, 4096, 4096), (1, 64, 1 << 17)):
        b = L.zgr_linear_i8_workspace(m, n, k)
        assert b >= m * ((k + 127) // 128 * 128) + 4 * m
    for bad in ((3, 8, (1 << 17) + 1), (-1, 8, 4), (1, 0, 4), (1, 8, 0), (1, 1 << 31, 4)):
        assert L.zgr_linear_i8_workspace(*bad) == zgr.EINVAL


@pytest.mark.parametrize("kw", [dict(x=None), dict(c=None), dict(s=None), dict(s=A + 1), dict(ldx=7), dict(ldc=7), dict(cols=0), dict(rows=-1), dict(rows=1 << 31), dict(dtype=5), dict(x=A + 2)])
def test_quantize_refuses(kw):
    a = dict(x=A, ldx=8, rows=4, cols=8, dtype=zgr.F32, c=A, ldc=8, s=A)
    a.update(kw)
    assert zgr.lib().zgr_quantize_rows(a["x"], a["ldx"], a["rows"], a["cols"], a["dtype"], a["c"], a["ldc"], a["s"], None) == zgr.EINVAL


GOOD = dict(x=A, ldx=64, w=A, ldw=64, ws=A, bias=None, r=None, ldr=0, y=A + (1 << 20), ldy=24, m=80, n=24, k=64, dtype=zgr.F32, p=0.0, space=A, space_bytes=1 << 20, xs=A)


@pytest.mark.parametrize("kw", [dict(x=None), dict(w=None), dict(ws=None), dict(y=None), dict(w=A + 8), dict(ldw=72), dict(ldw=48), dict(ldx=63), dict(ldy=23), dict(r=A, ldr=20),
                                dict(bias=A + 1), dict(ws=A + 2), dict(k=0), dict(k=(1 << 17) + 1), dict(n=0), dict(m=-1), dict(dtype=4), dict(p=-0.5), dict(p=float("nan")),
                                dict(space=None), dict(space=A + 4), dict(space_bytes=100), dict(ldw=1 << 40)])
def test_linear_refuses(kw):
    a = {**GOOD, **kw}
    rc = zgr.lib().zgr_linear_i8(a["x"], a["ldx"], a["w"], a["ldw"], a["ws"], a["bias"], a["r"], a["ldr"], a["y"], a["ldy"], a["m"], a["n"], a["k"], a["dtype"], a["p"], 0, 0,
                                 a["space"], a["space_bytes"], None)
    assert rc == zgr.EINVAL


@pytest.mark.parametrize("m", [1, 4, 80])
def test_a_product_refuses_its_tokens_as_the_output(m):
    # for a few tokens every block reads all of them while others write: the order would decide what it reads
    L, X = zgr.lib(), A + (1 << 20)
    assert L.zgr_linear_i8(X, 64, A, 64, A, None, X, 64, X, 64, m, 64, 64, zgr.F32, 0.0, 0, 0, A, 1 << 20, None) == zgr.EINVAL
    assert L.zgr_matmul_i8(X, 64, A, A, 64, A, None, None, 0, X, 64, m, 64, 64, zgr.F32, 0.0, 0, 0, None) == zgr.EINVAL


@pytest.mark.parametrize("kw", [dict(x=None), dict(xs=None), dict(xs=A + 2), dict(x=A + 8), dict(ldx=72), dict(ldx=1 << 40), dict(w=None), dict(k=0), dict(p=3.0)])
def test_matmul_refuses(kw):
    a = {**GOOD, **kw}
    rc = zgr.lib().zgr_matmul_i8(a["x"], a["ldx"], a["xs"], a["w"], a["ldw"], a["ws"], a["bias"], a["r"], a["ldr"], a["y"], a["ldy"], a["m"], a["n"], a["k"], a["dtype"], a["p"], 0, 0, None)
    assert rc == zgr.EINVAL


def test_status_wants_a_place():
    assert zgr.lib().zgr_linear_status(ctypes.POINTER(ctypes.c_int32)()) == zgr.EINVAL


def test_binding_refuses_tensors_of_the_host():
    import torch
    with pytest.raises((ValueError, RuntimeError)):       # (without a driver there is no current device to compare with)
        zgr.dropout(torch.zeros(4, 8), 0.1, 1)


def test_the_mask_of_the_64_bit_form():
    # hand-checked against the generator: element 8 o + i takes half i of block row * ceil(cols / 8) + o
    import oracle
    k = ref.keep(3, 10, 0.5, 123, 4)
    words = np.asarray(oracle.blocks(123, 4, ref.TAG_DROPOUT, 0, 6)).astype(np.uint32).reshape(6, 4)
    assert k[1, 9] == (int(words[1 * 2 + 1, 0] >> 16) >= 32768) and k[2, 5] == (int(words[2 * 2, 2] >> 16) >= 32768) and k[0, 4] == (int(words[0, 2] & 0xFFFF) >= 32768)
