"""Every form of the 8-bit product that sizes above a few tokens reach: pairs of CTAs and clusters of two and four, each with and without dropout,
residual and bias, in every type, against the 64-bit form; and the same bits from all of them.  tests/test_linear_plan.py asserts,
without a device, that these sizes reach the forms that are named here."""
import pytest
import torch

import forward_ref as ref
from paper_2601_12917_b200 import zgr
from test_gpu_linear_i8 import make

pytestmark = pytest.mark.gpu
DT = ref.DTYPES
PAIR, TILE = zgr.LINEAR_PAIR, zgr.LINEAR_TILE
# m, k, n, (kernel, tokens of a tile, CTAs of a tile): one chunk that is not full; the ends of tokens, of chunks and of 256 channels
PAIRS = [(257, 17, 20001, (PAIR, 96, 1)), (200, 1100, 20001, (PAIR, 128, 1)), (2100, 17, 5000, (PAIR, 192, 1))]
PAIRS_MORE = [(600, 1100, 9000, (PAIR, 160, 1)), (3000, 130, 5000, (PAIR, 224, 1)), (1500, 300, 12000, (PAIR, 256, 1))]
SPLIT = [(17, 1500, 40, (TILE, 16, 2)), (9, 1500, 129, (TILE, 16, 2)), (30, 2050, 40, (TILE, 16, 4)), (9, 2050, 129, (TILE, 16, 4)), (130, 2050, 257, (TILE, 16, 4)),
         (33, 1500, 9000, (TILE, 48, 2)), (70, 4100, 2000, (TILE, 48, 4)), (100, 4100, 3000, (TILE, 112, 4))]
# m, k, n by pairs, and (m, n) of parts of it by the other kernels
SAME_BITS = (200, 2050, 20001, [(1, 20001), (2, 300), (40, 20001), (30, 40), (100, 2000)])


def compare(m, k, n, plan, dtype, p, bias, residual):
    assert zgr.debug_linear_plan(m, n, k) == plan
    x, w = make((m, k), dtype), make((n, k), dtype, 1, 0.05)
    b = make((n,), dtype, 2) if bias else None
    r = make((m, n), dtype, 3) if residual else None
    wq, ws = zgr.quantize_rows(w)
    (ex, esx), (ew, esw) = ref.quantize(x.cpu().float().numpy()), ref.quantize(w.cpu().float().numpy())
    ey, size = ref.linear(ex, esx, ew, esw, p, 42, 6, ref.dbl(b), ref.dbl(r))
    y = zgr.linear_i8(x, wq, ws, bias=b, residual=r, p=p, seed=42, tensor=6)
    # conversion of the sum, product of the scales, product, bias, two of the dropout, residual
    ref.check(y, ey, size, dtype, 7, f"{m} {k} {n}")
    xq, xs = zgr.quantize_rows(x)
    assert torch.equal(zgr.matmul_i8(xq, xs, wq, ws, DT[dtype], bias=b, residual=r, p=p, seed=42, tensor=6), y)
    if residual:      # the result over the residual
        assert zgr.linear_i8(x, wq, ws, bias=b, residual=r, p=p, seed=42, tensor=6, out=r) is r and torch.equal(r, y)
    assert zgr.linear_status() == 0


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("p,bias,residual", [(0.0, True, False), (0.0, False, True), (0.3, False, False), (0.3, True, True), (1.0, True, True)])
@pytest.mark.parametrize("m,k,n,plan", PAIRS)
def test_pairs(m, k, n, plan, p, bias, residual, dtype):
    compare(m, k, n, plan, dtype, p, bias, residual)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("m,k,n,plan", PAIRS_MORE)
def test_pairs_of_other_tiles(m, k, n, plan, dtype):
    compare(m, k, n, plan, dtype, 0.25, True, dtype != "f16")


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("p,bias,residual", [(0.0, True, False), (0.0, False, True), (0.3, False, False), (0.3, True, True), (1.0, True, True)])
@pytest.mark.parametrize("m,k,n,plan", SPLIT)
def test_clusters(m, k, n, plan, p, bias, residual, dtype):
    compare(m, k, n, plan, dtype, p, bias, residual)


@pytest.mark.parametrize("residual", [False, True])
def test_a_result_has_the_same_bits_by_every_kernel(residual):
    # in fp32, where no rounding to the storage type hides a difference
    m, k, n, parts = SAME_BITS
    x, w, b = make((m, k), "f32"), make((n, k), "f32", 1, 0.05), make((n,), "f32", 2)
    r = make((m, n), "f32", 3) if residual else None
    wq, ws = zgr.quantize_rows(w)
    whole = zgr.linear_i8(x, wq, ws, bias=b, residual=r)
    for mm, nn in parts:
        for at in (0, m - mm):
            got = zgr.linear_i8(x[at:at + mm], wq[:nn], ws[:nn], bias=b[:nn], residual=None if r is None else r[at:at + mm, :nn])
            assert torch.equal(got, whole[at:at + mm, :nn]), (mm, nn, at)
    # with dropout, at the same number of channels
    whole = zgr.linear_i8(x, wq, ws, bias=b, residual=r, p=0.4, seed=3)
    for mm in (1, 2, 40, 130):
        got = zgr.linear_i8(x[:mm], wq, ws, bias=b, residual=None if r is None else r[:mm], p=0.4, seed=3)
        assert torch.equal(got, whole[:mm]), mm
