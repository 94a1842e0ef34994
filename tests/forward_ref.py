"""Plain 64-bit forms of the operators of the forward pass (dropout, row quantiser, 8-bit linear layer) and the bounds of their tests.

The generator is the oracle's; everything else is numpy in double precision from the definitions in zgr.h.

Bounds.  u = 2^-24 is half a step of fp32, h = finfo(dtype).eps / 2 half a step of the storage type (plus half the smallest subnormal).
Every fp32 operation is off by at most u of its result, so an expression of `ops` of them whose partial results are at most `size` in
magnitude is off by less than 1.01 ops u size, and its rounding to the storage type by h |y| more.
"""
import numpy as np
import torch

import oracle

TAG_DROPOUT = 2
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U32 = 2.0 ** -24
HALF_TINY = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}


def keep(rows, cols, p, seed, tensor):
    octets = -(-cols // 8)
    words = np.asarray(oracle.blocks(seed, tensor, TAG_DROPOUT, 0, rows * octets)).astype(np.uint32).reshape(-1, 4)
    halves = np.stack([words & 0xFFFF, words >> 16], axis=2).reshape(rows, octets * 8)
    return halves[:, :cols] >= int(np.rint(65536 * p))


def gain(p):
    t = int(np.rint(65536 * p))
    return 65536.0 / (65536 - t) if t < 65536 else 0.0


def dbl(t):
    return None if t is None else t.detach().cpu().double().numpy()


def dropout(x, p, seed, tensor, bias=None, residual=None):
    """(y, size): the result and the largest magnitude of a partial result, element by element; x etc. in double."""
    with np.errstate(invalid="ignore", over="ignore"):
        v = x if bias is None else x + bias
        size = np.abs(x) + (0 if bias is None else np.abs(bias))
        k = keep(x.shape[0], x.shape[1], p, seed, tensor)
        y = np.where(k, v * gain(p), 0.0)
        size = np.where(k, size * max(gain(p), 1.0), 0.0)
        if residual is not None:
            y, size = y + residual, size + np.abs(residual)
    return y, size


def quantize(x):
    """Codes (int64) and scales (float32), with the fp32 reciprocals and products that the definition names."""
    x = np.asarray(x, dtype=np.float32)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        a = np.abs(x).max(axis=1)
        bad = ~np.isfinite(x).all(axis=1)
        tiny = ~bad & (a < np.float32(2.0 ** -120))
        inv = np.where(bad | tiny, np.float32(0), (np.float32(1) / np.where(tiny, np.float32(1), a)).astype(np.float32) * np.float32(127)).astype(np.float32)
        codes = np.rint(np.where(bad[:, None], np.float32(0), x) * inv[:, None]).astype(np.int64)
        scale = np.where(tiny, np.float32(0), a * (np.float32(1) / np.float32(127))).astype(np.float32)
    scale[bad] = np.nan
    return codes, scale


def linear(qx, sx, qw, sw, p=0.0, seed=0, tensor=0, bias=None, residual=None):
    sums = qx.astype(np.float64) @ qw.astype(np.float64).T            # below 2^53: exact
    v = sums * (sx.astype(np.float64)[:, None] * sw.astype(np.float64)[None, :])
    if np.rint(65536 * p) == 0:
        y, size = v, np.abs(v)
        if bias is not None:
            y, size = y + bias, size + np.abs(bias)
        if residual is not None:
            y, size = y + residual, size + np.abs(residual)
        return y, size
    return dropout(v, p, seed, tensor, bias, residual)


def check(got, y, size, dtype, ops, what=""):
    """|got - y| within `ops` fp32 roundings of partial results up to `size` and the rounding to the storage type; NaN where y is NaN."""
    g = dbl(got)
    assert g.shape == y.shape, what
    h = torch.finfo(DTYPES[dtype]).eps / 2
    top = float(torch.finfo(DTYPES[dtype]).max)
    err = 1.01 * ops * U32 * size
    nan = np.isnan(y)
    assert np.array_equal(np.isnan(g), nan), f"{what}: NaN in other places"
    fits = ~nan & (np.abs(y) + err < top)            # beyond, the result rounds to infinity or the largest number
    tol = err + h * (np.abs(y) + err) + HALF_TINY[dtype]
    bad = np.abs(g[fits] - y[fits]) > tol[fits]
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off; worst {float((np.abs(g[fits] - y[fits]) / tol[fits]).max()):.2f} of the bound"
