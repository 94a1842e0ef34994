"""Dropout in the layouts and sizes that choose its other kernels: matrices whose rows start at different places of their 16-byte granules,
indexes of 64 bits, and the bias's gradient where its sums are exact."""
import numpy as np
import pytest
import torch

import forward_ref as ref
import oracle
from paper_2601_12917_b200 import zgr
from test_gpu_dropout import make

pytestmark = pytest.mark.gpu
DT = ref.DTYPES


class View:
    """rows x cols elements in a buffer of sevens, `pad` between the rows and `shift` in front of them."""
    def __init__(self, rows, cols, pad, shift, dtype, seed):
        self.buf = torch.full((rows * (cols + pad) + shift,), 7.0, dtype=DT[dtype], device="cuda")
        self.v = self.buf[shift:].view(rows, cols + pad)[:, :cols]
        self.v.copy_(make((rows, cols), dtype, seed))
        self.inside = torch.zeros_like(self.buf, dtype=torch.bool)
        self.inside[shift:].view(rows, cols + pad)[:, :cols] = True

    def untouched(self):
        return bool((self.buf[~self.inside] == 7.0).all())


def phase(t):
    return t.data_ptr() % 16


# groups of 1, 2, 4, ... 32 lanes a row, one to three groups; ends of octets and of groups; rows that share a warp and that do not fill the last
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("cols", [1, 2, 7, 8, 9, 15, 17, 31, 40, 63, 65, 100, 127, 129, 250, 257, 513, 600])
def test_rows_at_different_places_of_their_granules(cols, dtype):
    for rows, (px, sx), (pr, sr), (py, sy) in ((1, (0, 0), (0, 1), (0, 3)), (3, (2, 1), (0, 0), (5, 2)), (37, (1, 0), (3, 1), (2, 0)), (129, (0, 0), (1, 2), (9, 1))):
        x, r, y = View(rows, cols, px, sx, dtype, 1), View(rows, cols, pr, sr, dtype, 2), View(rows, cols, py, sy, dtype, 3)
        different = len({phase(t.v) for t in (x, r, y)} | {(t.v.stride(0) - x.v.stride(0)) % 8 for t in (r, y) if rows > 1}) > 1
        assert different
        b = make((cols,), dtype, 4)
        for bias, residual, p in ((None, r.v, 0.3), (b, r.v, 0.3), (b, None, 0.7), (None, None, 0.5), (b, r.v, 0.0), (b, r.v, 1.0)):
            assert zgr.dropout(x.v, p, 21, 3, bias=bias, residual=residual, out=y.v) is y.v
            ey, size = ref.dropout(ref.dbl(x.v), p, 21, 3, ref.dbl(bias), ref.dbl(residual))
            ref.check(y.v, ey, size, dtype, 4, f"{rows} x {cols} p {p}")
        dx = zgr.dropout_backward(x.v, 0.3, 21, 3, out=y.v)
        ex, size = ref.dropout(ref.dbl(x.v), 0.3, 21, 3)
        ref.check(dx, ex, size, dtype, 2)
        dx2, db = zgr.dropout_backward(x.v, 0.3, 21, 3, bias_grad=True, out=y.v)
        assert torch.equal(dx2, zgr.dropout_backward(x.v, 0.3, 21, 3))
        ref.check(db, ex.sum(axis=0), size.sum(axis=0), dtype, rows + 2)
        want = zgr.dropout(x.v, 0.4, 5, 1, bias=b, residual=r.v)
        zgr.dropout(x.v, 0.4, 5, 1, bias=b, residual=r.v, out=r.v)      # over the residual, whose rows lie otherwise than those of x
        assert torch.equal(r.v, want)
        want = zgr.dropout(x.v, 0.4, 5, 1, residual=y.v)
        zgr.dropout(x.v, 0.4, 5, 1, residual=y.v, out=x.v)              # over x
        assert torch.equal(x.v, want)
        assert x.untouched() and r.untouched() and y.untouched()


def exact_sums(rows, cols, dtype, p, pad=0, shift=0, holes=False):
    # whole numbers of at most 3 and a scale of 1 or 2: sums stay far below 2^24, so every order of additions gives the same fp32 number
    g = torch.Generator().manual_seed(rows + 7 * cols)
    values = torch.randint(-3, 4, (rows, cols), generator=g).double().numpy()
    k = ref.keep(rows, cols, p, 17, 9)
    buf = torch.zeros(rows * (cols + pad) + shift, dtype=DT[dtype], device="cuda")
    dy = buf[shift:].view(rows, cols + pad)[:, :cols]
    held = torch.from_numpy(values)
    if holes:             # what is dropped contributes nothing, whatever it holds
        held = torch.where(torch.from_numpy(k), held, torch.where(torch.arange(cols) % 2 == 0, float("nan"), float("-inf")).double())
    dy.copy_(held.to(DT[dtype]).cuda())
    want = np.where(k, values * ref.gain(p), 0.0)
    dx, db = zgr.dropout_backward(dy, p, 17, 9, bias_grad=True)
    assert np.array_equal(ref.dbl(dx), want)
    assert torch.equal(db, torch.from_numpy(want.sum(axis=0)).to(DT[dtype]).cuda())
    dx, db2 = zgr.dropout_backward(dy, p, 17, 9, bias_grad=True, out=dy)      # over dy
    assert np.array_equal(ref.dbl(dx), want) and torch.equal(db2, db)


# one range of rows and several; rows a thread and the rest of them; narrow matrices whose rows share a warp
@pytest.mark.parametrize("p", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,cols", [(1, 1), (7, 9), (130, 64), (129, 300), (600, 300), (4097, 3), (4096, 8), (5000, 16), (1100, 24), (513, 63), (2371, 1024), (9000, 129), (20011, 1)])
def test_sums_of_the_bias_are_exact(rows, cols, dtype, p):
    exact_sums(rows, cols, dtype, p)
    if rows <= 5000:
        exact_sums(rows, cols, dtype, p, pad=3, shift=1)
        exact_sums(rows, cols, dtype, p, holes=p > 0)
        exact_sums(rows, cols, dtype, p, pad=-cols % 8, holes=p > 0)      # rows on 16-byte boundaries, their ends not whole octets


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("p", [0.1, 0.37, 0.9])
@pytest.mark.parametrize("rows,cols", [(130, 129), (4097, 3), (600, 1000), (3000, 520)])
def test_sums_of_the_bias_of_normals(rows, cols, p, dtype):
    x = make((rows, cols), dtype)
    dx, db = zgr.dropout_backward(x, p, 99, 3, bias_grad=True)
    ex, size = ref.dropout(ref.dbl(x), p, 99, 3)
    ref.check(dx, ex, size, dtype, 2)
    # The longest chain of additions: a thread's rows, its block's row lanes, every eighth range and the eight sums of them.  A block has 256
    # threads and a row takes 1 to 32 of them; there are as many ranges as the workspace has rows (one if there is none).
    lanes = 256 // min(32, 1 << (-(-cols // 8) - 1).bit_length())
    ranges = max(1, zgr.lib().zgr_dropout_backward_workspace(rows, cols) // (4 * cols))
    chain = -(-rows // (ranges * lanes)) + 1 + lanes + -(-ranges // 8) + 8
    assert ranges == 1 or chain < rows
    ref.check(db, ex.sum(axis=0), size.sum(axis=0), dtype, chain + 2)


def halves(seed, tensor, first, n):
    words = np.asarray(oracle.blocks(seed, tensor, ref.TAG_DROPOUT, first, n)).astype(np.uint32).reshape(-1, 4)
    return np.stack([words & 0xFFFF, words >> 16], axis=2).reshape(-1, 8)


@pytest.fixture
def free_memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


PLACES = (0, 12345, (1 << 31) - 2, (1 << 31) - 1)      # and the last rows


def check_rows(y, cols, keep_from, seed, tensor, kept, n=100):
    rows = y.shape[0]
    for first in {f for f in PLACES + ((1 << 32) - 2, rows - n) if f + n <= rows}:
        k = halves(seed, tensor, first, n)[:, :cols] >= keep_from
        assert np.array_equal(y[first:first + n].float().cpu().numpy(), np.where(k, kept, 0.0)), first


def test_more_than_31_bits_of_short_rows(free_memory):
    rows = (1 << 31) + 205
    # one column, off the boundaries: a piece a row
    y = torch.ones(rows, 1, dtype=torch.float16, device="cuda")
    zgr.dropout(y, 0.5, 8, 2, residual=y, out=y)
    check_rows(y - 1, 1, 32768, 8, 2, 2.0)
    zgr.dropout(y.fill_(1), 0.5, 9, 2, out=y)
    check_rows(y, 1, 32768, 9, 2, 2.0)
    del y
    # whole octets with a bias
    y = torch.ones(rows, 8, dtype=torch.float16, device="cuda")
    b = torch.arange(8, dtype=torch.float16, device="cuda")
    zgr.dropout(y, 0.5, 8, 2, bias=b, out=y)
    check_rows(y, 8, 32768, 8, 2, 2.0 * (1 + np.arange(8)))


@pytest.mark.parametrize("cols", [1, 8])
def test_bias_gradient_of_more_than_32_bits_of_rows(cols, free_memory):
    # block numbers of 64 bits, with rows anywhere and on the boundaries
    rows = (1 << 32) + 205
    dy = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    dx, db = zgr.dropout_backward(dy, 0.5, 8, 2, bias_grad=True, out=dy)
    check_rows(dx, cols, 32768, 8, 2, 2.0)
    want = sum(part.sum(dim=0, dtype=torch.float64) for part in dx.split(1 << 26))
    # 592 ranges of 7.3 million rows: a range's sum is a whole number below 2^24, exact; then eight chains of 74 additions and 8 more, and bf16
    assert bool(((db.double() - want).abs() <= want * (82 * 2.0 ** -24 * 1.01 + 2.0 ** -8)).all())
    assert bool(((want / rows - 1).abs() < 5 / rows ** 0.5).all())       # (twice the share that is kept: five standard deviations)
