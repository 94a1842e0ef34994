"""Dropout from the counter-based generator: forward, backward, the bias's gradient, against the 64-bit form; layouts, masks, graphs, refusals."""
import threading

import numpy as np
import pytest
import torch

import forward_ref as ref
import oracle
from paper_2601_12917_b200 import zgr

pytestmark = pytest.mark.gpu
DT = ref.DTYPES
# one element to several octets, ends of octets, rows of 1, 8, 32 and more octets, several blocks of 256 threads, the line between the
# one-octet and the four-octet form (148 * 8 * 256 octets), column sums by one range of rows and by several
SHAPES = [(1, 1), (1, 7), (3, 8), (5, 9), (2, 256), (7, 255), (33, 40), (4, 1000), (3, 4096), (130, 129), (1, 70001), (2371, 1024), (600, 4100),
          (128, 300), (129, 300), (4096, 3), (4097, 3), (300, 64), (1100, 24), (513, 63)]


def make(shape, dtype, seed=0, sigma=1.0):
    g = torch.Generator().manual_seed(seed + 31 * shape[-1])
    return (torch.randn(shape, generator=g) * sigma).to(DT[dtype]).cuda()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_and_backward(shape, dtype):
    rows, cols = shape
    for bias, residual, p in ((False, False, 0.1), (True, True, 0.5), (True, False, 0.37), (False, True, 0.9)):
        x, b = make(shape, dtype), make((cols,), dtype, 1) if bias else None
        r = make(shape, dtype, 2) if residual else None
        y = zgr.dropout(x, p, 12345678901234567, 7, bias=b, residual=r)
        ey, size = ref.dropout(ref.dbl(x), p, 12345678901234567, 7, ref.dbl(b), ref.dbl(r))
        ref.check(y, ey, size, dtype, 4, f"{shape} {bias} {residual}")
    dx, db = zgr.dropout_backward(x, p, 99, 3, bias_grad=True)
    ex, size = ref.dropout(ref.dbl(x), p, 99, 3)
    ref.check(dx, ex, size, dtype, 2, f"{shape} dx")
    # each term off by 2 u, each of at most rows additions by u of a partial sum: below (rows + 2) u of the sum of magnitudes
    ref.check(db, ex.sum(axis=0), size.sum(axis=0), dtype, rows + 2, f"{shape} dbias")
    assert torch.equal(dx, zgr.dropout_backward(x, p, 99, 3))
    again = zgr.dropout_backward(x, p, 99, 3, bias_grad=True)
    assert torch.equal(again[0], dx) and torch.equal(again[1], db)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,cols,pad,shift", [(9, 64, 8, 0), (9, 64, 1, 0), (9, 61, 3, 0), (5, 512, 0, 1), (17, 300, 4, 4), (6, 24, 40, 3), (3, 16, 16, 8)])
def test_strides_and_alignment(rows, cols, pad, shift, dtype):
    # views into a larger buffer, whose other elements stay as they were; the mask does not know of either
    def view(fill, seed):
        buf = torch.full((rows * (cols + pad) + shift,), fill, dtype=DT[dtype], device="cuda")
        v = buf[shift:].view(rows, cols + pad)[:, :cols]
        v.copy_(make((rows, cols), dtype, seed))
        return buf, v
    xb, x = view(7.0, 0)
    rb, r = view(7.0, 1)
    yb, y = view(7.0, 2)
    b = make((cols + 1,), dtype, 3)[1:]
    want = zgr.dropout(x.contiguous(), 0.3, 5, 1, bias=b.clone(), residual=r.contiguous())
    zgr.dropout(x, 0.3, 5, 1, bias=b, residual=r, out=y)
    assert torch.equal(y, want)
    outside = torch.ones_like(yb, dtype=torch.bool)
    outside[shift:].view(rows, cols + pad)[:, :cols] = False
    for buf in (xb, rb, yb):
        assert bool((buf[outside] == 7.0).all())
    dwant, bwant = zgr.dropout_backward(r.contiguous(), 0.3, 5, 1, bias_grad=True)
    dgot, bgot = zgr.dropout_backward(r, 0.3, 5, 1, bias_grad=True, out=x)
    assert torch.equal(dgot, dwant) and bool((xb[outside] == 7.0).all())
    # (rows that start anywhere are summed by other lanes: same terms, another order)
    ex, size = ref.dropout(ref.dbl(r), 0.3, 5, 1)
    ref.check(bgot, ex.sum(axis=0), size.sum(axis=0), dtype, rows + 2)


def test_probabilities_and_masked_values():
    x = make((64, 1000), "f32")
    assert torch.equal(zgr.dropout(x, 0.0, 1), x) and torch.equal(zgr.dropout(x, 2.0 ** -18, 1), x)     # below half a step: nothing is dropped
    assert bool((zgr.dropout(x, 1.0, 1) == 0).all())
    x[:, ::3] = float("inf")
    x[:, 1::3] = float("nan")
    for p, bias in ((1.0, None), (0.5, torch.full((1000,), float("nan"), device="cuda"))):
        y = zgr.dropout(x, p, 1, bias=bias, residual=torch.ones_like(x))
        dropped = torch.from_numpy(~ref.keep(64, 1000, p, 1, 0)).cuda()
        assert bool((y[dropped] == 1).all()) and bool((~torch.isfinite(y[~dropped])).all())
    # the share that is kept, over 2^22 elements: five standard deviations
    for p in (0.1, 0.5, 0.95):
        y = zgr.dropout(torch.ones(1, 1 << 22, device="cuda"), p, 4)
        q = 1 - round(65536 * p) / 65536
        assert abs(float((y != 0).double().mean()) - q) < 5 * (q * (1 - q) / (1 << 22)) ** 0.5
        assert float((y - 1 / q)[y != 0].abs().max()) < 1e-5 / q
    # other seeds, tensors: other masks; the same: the same, in every type
    a = zgr.dropout(torch.ones(8, 512, device="cuda"), 0.5, 4, 1)
    for seed, tensor in ((5, 1), (4, 2), (4 + (1 << 32), 1)):
        assert 0.4 < float((zgr.dropout(torch.ones(8, 512, device="cuda"), 0.5, seed, tensor) != a).double().mean()) < 0.6
    for dt in DT.values():
        assert torch.equal(zgr.dropout(torch.ones(8, 512, device="cuda", dtype=dt), 0.5, 4, 1) != 0, a != 0)


def test_mask_is_the_generators_third_stream():
    z = zgr.Zgr([torch.zeros(4, device="cuda")], [None], 1.0, 1e-3)
    words = z.debug_philox(77, 5, zgr.TAG_DROPOUT, 0, 512).cpu().numpy().astype(np.uint32)
    halves = np.stack([words & 0xFFFF, words >> 16], axis=2).reshape(64, 64)
    y = zgr.dropout(torch.ones(64, 64, device="cuda"), 0.25, 77, 5)
    assert np.array_equal(y.cpu().numpy() != 0, halves >= 16384)


def test_in_place_and_more_dimensions():
    x = make((4, 6, 80), "bf16")
    r = make((4, 6, 80), "bf16", 1)
    want = zgr.dropout(x.view(24, 80), 0.2, 3, residual=r.view(24, 80)).view(4, 6, 80)
    assert torch.equal(zgr.dropout(x, 0.2, 3, residual=r), want)
    x2, r2 = x.clone(), r.clone()
    assert torch.equal(zgr.dropout(x2, 0.2, 3, residual=r, out=x2), want) and torch.equal(zgr.dropout(x, 0.2, 3, residual=r2, out=r2), want)
    assert torch.equal(zgr.dropout_backward(x, 0.2, 3), zgr.dropout_backward(x.clone(), 0.2, 3, out=x.clone()))
    empty = torch.empty(0, 80, device="cuda")
    assert zgr.dropout(empty, 0.2, 3).shape == (0, 80) and zgr.dropout(torch.empty(5, 0, device="cuda"), 0.2, 3).shape == (5, 0)
    d, b = zgr.dropout_backward(empty, 0.2, 3, bias_grad=True)
    assert d.shape == (0, 80) and bool((b == 0).all())


def test_gradient_against_differences():
    # the loss sum(c * y) is linear in x and bias: its differences are exact up to the rounding of the sums, here in fp32
    x, b, c = make((6, 24), "f32"), make((24,), "f32", 1), make((6, 24), "f32", 2)
    def loss(x, b):
        return float((zgr.dropout(x, 0.4, 8, 2, bias=b).double() * c.double()).sum())
    dx, db = zgr.dropout_backward(c, 0.4, 8, 2, bias_grad=True)
    base = loss(x, b)
    for i in range(0, 144, 11):
        moved = x.clone()
        moved.view(-1)[i] += 1.0
        # y is off by at most 2 u |y| on each side: 4 u (|x| + 2) |c| / (1 - p)
        assert abs(loss(moved, b) - base - float(dx.view(-1)[i])) < 4 * ref.U32 * 8 * 5 / 0.6
    for i in range(0, 24, 5):
        moved = b.clone()
        moved[i] += 1.0
        assert abs(loss(x, moved) - base - float(db[i])) < 6 * 4 * ref.U32 * 8 * 5 / 0.6


def test_streams_and_graphs():
    x = make((300, 1000), "f16")
    want = zgr.dropout(x, 0.3, 11, 4)
    dwant, bwant = zgr.dropout_backward(x, 0.3, 11, 4, bias_grad=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = zgr.dropout(x, 0.3, 11, 4, stream=side)
    dgot = zgr.dropout_backward(x, 0.3, 11, 4, bias_grad=True, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(dgot[0], dwant) and torch.equal(dgot[1], bwant)
    graphs = []
    for _ in range(2):                                   # two graphs at once, each with a workspace of its own
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = zgr.dropout(x, 0.3, 11, 4)
            d, b = zgr.dropout_backward(x, 0.3, 11, 4, bias_grad=True)
        graphs.append((g, out, d, b))
    keep = x.clone()
    x.zero_()
    streams = [torch.cuda.Stream() for _ in graphs]
    x.copy_(keep)
    torch.cuda.synchronize()
    for (g, *_), s in zip(graphs, streams):
        with torch.cuda.stream(s):
            for _ in range(3):
                g.replay()
    torch.cuda.synchronize()
    for _, out, d, b in graphs:
        assert torch.equal(out, want) and torch.equal(d, dwant) and torch.equal(b, bwant)


def test_binding_refuses():
    x = make((4, 16), "f32")
    for bad in (lambda: zgr.dropout(x.cpu(), 0.1, 1), lambda: zgr.dropout(x.double(), 0.1, 1), lambda: zgr.dropout(x.t(), 0.1, 1),
                lambda: zgr.dropout(x, 0.1, 1, residual=x[:2]), lambda: zgr.dropout(x, 0.1, 1, residual=x.half()), lambda: zgr.dropout(x, 0.1, 1, bias=x[0, :8]),
                lambda: zgr.dropout(x, 0.1, 1, bias=torch.zeros(32, device="cuda")[::2]), lambda: zgr.dropout(x, 0.1, 1, out=x.half()),
                lambda: zgr.dropout(x.view(2, 2, 16).transpose(0, 1), 0.1, 1), lambda: zgr.dropout(x.sum(), 0.1, 1), lambda: zgr.dropout_backward(x.t(), 0.1, 1)):
        with pytest.raises(ValueError):
            bad()
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(zgr.ZgrError) as e:
            zgr.dropout(x, p, 1)
        assert e.value.code == zgr.EINVAL
    with pytest.raises(zgr.ZgrError):
        zgr.dropout(x[:1].expand(4, 16), 0.1, 1)         # rows on top of each other


def keep_blocks(seed, tensor, first, n):
    words = np.asarray(oracle.blocks(seed, tensor, ref.TAG_DROPOUT, first, n)).astype(np.uint32).reshape(-1, 4)
    return np.stack([words & 0xFFFF, words >> 16], axis=2).reshape(-1) >= 32768


@pytest.mark.parametrize("cols", [61440, 61441])
def test_offsets_past_32_bits(cols):
    # more than 2^32 elements: the last rows against the generator's blocks for them (octets by a 64-bit division from 2^31 on)
    rows = (1 << 32) // cols + 3
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 1 << 32
    y = zgr.dropout(x, 0.5, 21, 3, out=x)
    octets = (cols + 7) // 8
    for row in (0, 35000, rows - 2, rows - 1):
        assert np.array_equal(y[row].float().cpu().numpy(), np.where(keep_blocks(21, 3, row * octets, octets)[:cols], 2.0, 0.0))


@pytest.mark.parametrize("cols", [(1 << 31) + 64, (1 << 31) + 13])
def test_rows_longer_than_31_bits(cols):
    x = torch.ones(cols, dtype=torch.float16, device="cuda")
    b = torch.zeros(cols, dtype=torch.float16, device="cuda") if cols % 8 == 0 else None
    for bias in (None, b) if b is not None else (None,):
        y = zgr.dropout(x, 0.5, 4, 2, bias=bias)
        last = (cols + 7) // 8 - 100
        keep = keep_blocks(4, 2, last, 100)[:cols - 8 * last]
        assert np.array_equal(y[8 * last:].float().cpu().numpy(), np.where(keep, 2.0, 0.0))
        assert np.array_equal(y[:800].float().cpu().numpy(), np.where(keep_blocks(4, 2, 0, 100), 2.0, 0.0))


def test_a_chain_of_launches_sees_what_is_in_front_of_it():
    # every call starts while the one in front ends, and works in place on what that one writes: the same as with a wait behind each
    def chain(wait):
        x = make((37, 1021), "f32", 5)
        b = make((1021,), "f32", 6)
        for i in range(60):
            zgr.dropout(x, 0.05, i, bias=b, out=x)
            if wait:
                torch.cuda.synchronize()
            d, b = zgr.dropout_backward(x, 0.1, i, bias_grad=True, out=x)
            if wait:
                torch.cuda.synchronize()
            zgr.dropout(d, 0.2, i, 1, residual=d, out=x)
            x.mul_(0.5)
            b.mul_(0.1)
        return x, b
    quick, slow = chain(False), chain(True)
    assert torch.equal(quick[0], slow[0]) and torch.equal(quick[1], slow[1])


def test_calls_from_several_threads():
    want = [zgr.dropout(make((64, 999), "f16", i), 0.3, i) for i in range(4)]
    torch.cuda.synchronize()
    got, streams = [[] for _ in range(4)], [torch.cuda.Stream() for _ in range(4)]

    def work(i):
        x = make((64, 999), "f16", i)
        torch.cuda.synchronize()
        for _ in range(50):
            got[i].append(zgr.dropout(x, 0.3, i, stream=streams[i]))
        streams[i].synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for w, ys in zip(want, got):
        assert len(ys) == 50 and all(torch.equal(w, y) for y in ys)


def test_outputs_count_as_written_and_pending_signs_are_refused():
    x = make((6, 16), "f32").requires_grad_()
    y = (x * x).sum()
    zgr.dropout(x.detach(), 0.5, 1)
    zgr.dropout_backward(x.detach(), 0.5, 1)
    y.backward(retain_graph=True)
    for write in (lambda: zgr.dropout(x.detach(), 0.5, 1, out=x.detach()), lambda: zgr.dropout_backward(x.detach(), 0.5, 1, out=x.detach())):
        y = (x * x).sum()
        write()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    with torch.inference_mode():
        z = make((6, 16), "f32")
        assert zgr.dropout(z, 0.5, 1, out=z) is z
    assert zgr.dropout(z, 0.5, 1, out=z) is z
    with pytest.raises(ValueError):
        zgr.dropout(x.detach()._neg_view(), 0.5, 1)
