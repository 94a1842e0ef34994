"""Row quantiser and 8-bit linear layer against the 64-bit form: sizes around tiles, chunks and codes' ends, every epilogue, layouts,
values that are not finite, graphs, refusals, and the run of them with a sweep between."""
import threading

import numpy as np
import pytest
import torch

import forward_ref as ref
import oracle
from paper_2601_12917_b200 import zgr

pytestmark = pytest.mark.gpu
DT = ref.DTYPES


def make(shape, dtype, seed=0, sigma=1.0):
    g = torch.Generator().manual_seed(seed + 31 * shape[-1] + shape[0])
    return (torch.randn(shape, generator=g) * sigma).to(DT[dtype]).cuda()


def codes_of(t):
    return t.cpu().numpy().astype(np.int64)


# one warp a row up to 1536 elements, four up to 6144, eight up to 12288, twelve up to 18432, then the form that reads twice; octets a thread
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 7), (9, 8), (3, 33), (130, 64), (7, 1000), (2, 1024), (3, 1025), (4, 1536), (5, 1537), (3, 2049), (5, 4096), (2, 4099), (3, 6144), (2, 6145), (3, 8192), (2, 11008), (2, 12289), (2, 16384), (2, 18432), (2, 18433), (1, 50265)])
def test_quantize_rows(rows, cols, dtype):
    x = make((rows, cols), dtype)
    if rows > 2:
        x[1] = 0
        x[2, cols // 2] = float("-inf") if rows % 2 else float("nan")
    for src, pitch in ((x, None), (x, cols), (torch.cat([x, x], 1)[:, :cols] if cols % 8 else x, None), (torch.cat([x[:, :1], x], 1)[:, 1:], cols + 3)):
        codes, scales = zgr.quantize_rows(src, pitch=pitch)
        ec, es = ref.quantize(x.cpu().float().numpy())
        assert np.array_equal(codes_of(codes), ec)
        assert np.array_equal(scales.cpu().numpy(), es, equal_nan=True)
        line = 16 if cols < 512 else 128
        assert codes.stride(0) == ((cols + line - 1) // line * line if pitch is None else pitch)


def test_quantize_small_and_large_values():
    x = torch.tensor([[2.0 ** -120, 0, -(2.0 ** -121)], [2.0 ** -121, 2.0 ** -122, 0], [1e-45, 0, 0], [3.4e38, -3.4e38, 1e38], [127, 63.5, 0.5], [1.5, -2.5, 127]], device="cuda")
    codes, scales = zgr.quantize_rows(x)
    ec, es = ref.quantize(x.cpu().numpy())
    assert np.array_equal(codes_of(codes), ec) and np.array_equal(scales.cpu().numpy(), es)
    assert ec.tolist() == [[127, 0, -64], [0, 0, 0], [0, 0, 0], [127, -127, 37], [127, 64, 0], [2, -2, 127]]


def test_quantized_rows_are_the_compressed_coefficients():
    # the sender's half of the DTC codes: what the library quantises it sweeps with, as the oracle does with these codes
    rows, cols, r = 96, 200, 16
    w = make((rows, cols), "f32", 1, 0.02)
    U = torch.linalg.qr(torch.randn(rows, r, dtype=torch.float64, generator=torch.Generator().manual_seed(3)))[0].float().cuda().contiguous()
    G = make((r, cols), "f32", 2)
    codes, scales = zgr.quantize_rows(G, pitch=cols)
    eq, es, _ = oracle.dtc_quantise(ref.dbl(G), 8, True)
    assert (np.abs(scales.cpu().numpy().astype(np.float64) / es - 1) <= 2.0 ** -23).all()      # (a reciprocal and a product, the oracle has one quotient)
    assert np.abs(codes_of(codes) - eq).max() <= 1                     # (the oracle divides by the scale; a tie may fall to the other side)
    z = zgr.Zgr([w], [U], 0.0, 1e-3)
    z.set_coeffs_dtc(0, codes, scales)
    before = ref.dbl(w)
    a, b = z.scalars()
    z.perturb(9, 1.0)
    deq = codes_of(codes) * scales.cpu().numpy().astype(np.float64)[:, None]
    want = before + b * (ref.dbl(U) @ deq)
    assert np.abs(ref.dbl(w) - want).max() <= 1e-6 * np.abs(want).max() + 2e-6 * b * np.abs(ref.dbl(U)).max() * np.abs(deq).max()


def run_case(m, k, n, dtype, p, bias, residual, seed=0):
    x, w = make((m, k), dtype, seed), make((n, k), dtype, seed + 1, 0.05)
    b = make((n,), dtype, seed + 2) if bias else None
    r = make((m, n), dtype, seed + 3) if residual else None
    wq, ws = zgr.quantize_rows(w)
    y = zgr.linear_i8(x, wq, ws, bias=b, residual=r, p=p, seed=42, tensor=6)
    xq, xs = zgr.quantize_rows(x)
    y2 = zgr.matmul_i8(xq, xs, wq, ws, DT[dtype], bias=b, residual=r, p=p, seed=42, tensor=6)
    ex, esx = ref.quantize(x.cpu().float().numpy())
    ew, esw = ref.quantize(w.cpu().float().numpy())
    ey, size = ref.linear(ex, esx, ew, esw, p, 42, 6, ref.dbl(b), ref.dbl(r))
    # conversion of the sum, product of the scales, product, bias, two of the dropout, residual
    ref.check(y, ey, size, dtype, 7, f"linear {m} {k} {n}")
    ref.check(y2, ey, size, dtype, 7, f"matmul {m} {k} {n}")
    assert zgr.linear_status() == 0
    return x, wq, ws, y


# m: few tokens, a row of accumulators of 16, the ends of it, several; k: one code, the ends of 16 and 128, several chunks, enough for every
# split; n: one channel, the ends of 8, 32 and 128
@pytest.mark.parametrize("m,k,n", [(1, 1, 1), (1, 16, 7), (2, 17, 33), (3, 100, 129), (4, 513, 40), (5, 16, 8), (7, 127, 130), (9, 129, 31), (16, 128, 128), (17, 640, 257),
                                   (31, 1024, 100), (33, 2048, 64), (64, 4096, 130), (100, 1000, 300), (128, 384, 256), (129, 512, 640), (255, 136, 65),
                                   (256, 256, 256), (257, 300, 384), (300, 1027, 200), (520, 2050, 140), (1, 4096, 1000), (8, 11008, 520), (4, 24000, 64), (4, 24600, 64), (2000, 300, 2500), (1030, 1100, 2100), (3, 6000, 9000), (16, 6145, 20000),
                                   (15, 12200, 5000), (16, 16000, 6000), (13, 1000, 19000),
                                   (3, 4100, 2048), (3, 4100, 2040), (5, 4100, 1024), (8, 4100, 1020), (6, 300, 700), (8, 11000, 300), (7, 31, 50), (4, 40, 8192), (5, 40, 8193)])
@pytest.mark.parametrize("dtype", list(DT))
def test_linear_sizes(m, k, n, dtype):
    run_case(m, k, n, dtype, 0.0, n % 2 == 0, m % 2 == 0)


@pytest.mark.parametrize("m", [1, 2, 3, 4, 6, 8, 9, 20, 300])
@pytest.mark.parametrize("p,bias,residual", [(0.0, True, False), (0.3, False, False), (0.3, True, True), (1.0, True, True), (0.9, False, True)])
def test_linear_epilogues(m, p, bias, residual):
    run_case(m, 200, 150, "bf16", p, bias, residual, 5)
    run_case(m, 640, 136, "f32", p, bias, residual, 6)


def test_largest_sums_are_exact():
    # codes of +-127 throughout: 127 * 127 * 2^17 fits 32 bits; sums of one row differ from those of its neighbour by one product
    k = 1 << 17
    for m in (1, 5):
        xq = torch.full((m, k), 127, dtype=torch.int8, device="cuda")
        wq = torch.full((3, k), 127, dtype=torch.int8, device="cuda")
        wq[1] = -127
        wq[2, 5] = 126
        one_m, one_n = torch.ones(m, device="cuda"), torch.ones(3, device="cuda")
        y = zgr.matmul_i8(xq, one_m, wq, one_n, torch.float32)
        top = 127 * 127 * k
        want = torch.tensor([float(np.float32(top)), -float(np.float32(top)), float(np.float32(top - 127))], device="cuda")
        assert torch.equal(y, want.expand(m, 3))
    x = torch.full((1, k), 2.0, device="cuda")
    y = zgr.linear_i8(x, wq, one_n)
    assert float(y[0, 0]) == float(np.float32(np.float32(top) * (np.float32(2) * (np.float32(1) / np.float32(127)))))


def test_strides_alignment_and_what_lies_around():
    for m in (1, 3, 40):
        k, n = 200, 70
        xb = torch.full((m * 230 + 3,), float("nan"), dtype=torch.bfloat16, device="cuda")
        x = xb[3:].view(m, 230)[:, :k]
        x.copy_(make((m, k), "bf16"))
        w = make((n, k), "bf16", 1)
        wq, ws = zgr.quantize_rows(w)
        wide = torch.full((n, 272), 99, dtype=torch.int8, device="cuda")      # codes behind the k-th of a row are not used
        wide[:, :k] = wq
        yb = torch.full((m * 81 + 1,), 7.0, dtype=torch.bfloat16, device="cuda")
        y = yb[1:].view(m, 81)[:, :n]
        rb = torch.full((m * 75,), float("nan"), dtype=torch.bfloat16, device="cuda")
        r = rb.view(m, 75)[:, 2:72]
        r.copy_(make((m, n), "bf16", 2))
        want = zgr.linear_i8(x.contiguous(), wq, ws, residual=r.contiguous(), p=0.2, seed=3)
        zgr.linear_i8(x, wide[:, :k], ws, residual=r, p=0.2, seed=3, out=y)
        assert torch.equal(y, want)
        outside = torch.ones_like(yb, dtype=torch.bool)
        outside[1:].view(m, 81)[:, :n] = False
        assert bool((yb[outside] == 7.0).all())
        zgr.linear_i8(x, wide[:, :k], ws, residual=r, p=0.2, seed=3, out=r)   # the result over the residual
        assert torch.equal(r, want)
        x3 = x.contiguous().view(1, m, k)
        assert torch.equal(zgr.linear_i8(x3, wq, ws, residual=want.view(1, m, n)), zgr.linear_i8(x.contiguous(), wq, ws, residual=want).view(1, m, n))


def test_values_that_are_not_finite():
    for m in (2, 30):
        x, w = make((m, 96), "f16"), make((40, 96), "f16", 1)
        wq, ws = zgr.quantize_rows(w)
        clean = zgr.linear_i8(x, wq, ws, p=0.5, seed=2)
        x[0, 3] = float("inf")
        x[1] = 0
        y = zgr.linear_i8(x, wq, ws, p=0.5, seed=2)
        k = torch.from_numpy(ref.keep(m, 40, 0.5, 2, 0)).cuda()
        assert bool(torch.isnan(y[0][k[0]]).all()) and bool((y[0][~k[0]] == 0).all()) and bool((y[1] == 0).all())
        assert torch.equal(y[2:], clean[2:])
        w[5, 0] = float("nan")
        wq, ws = zgr.quantize_rows(w)
        y = zgr.linear_i8(x, wq, ws)
        assert bool(torch.isnan(y[:, 5]).all()) and bool(torch.isfinite(y[1:, :5]).all())


def test_a_token_does_not_depend_on_the_batch():
    # every kernel: the same token gives the same bits alone and in any batch (sums are exact, the epilogue is the same arithmetic)
    x, w = make((600, 1000), "f32"), make((200, 1000), "f32", 1)
    wq, ws = zgr.quantize_rows(w)
    b = make((200,), "f32", 2)
    whole = zgr.linear_i8(x, wq, ws, bias=b)
    for m in (1, 2, 3, 4, 5, 16, 17, 100, 257):
        same = torch.equal(zgr.linear_i8(x[:m], wq, ws, bias=b), whole[:m])
        assert same, m


def test_block_of_a_forward_pass_between_two_sweeps():
    # perturb, requantise, layer with dropout and residual; twice, for L+ and L-, under one mask; against the 64-bit form
    W = make((256, 320), "bf16", 1, 0.05)
    U = torch.linalg.qr(torch.randn(256, 16, dtype=torch.float64, generator=torch.Generator().manual_seed(3)))[0].float().cuda().contiguous()
    z = zgr.Zgr([W], [U], 0.5, 1e-2)
    x, h = make((48, 320), "bf16", 2), make((48, 256), "bf16", 3)
    for scale in (1e-2, -2e-2):
        z.perturb(5, scale)
        wq, ws = zgr.quantize_rows(W)
        y = zgr.linear_i8(x, wq, ws, residual=h, p=0.25, seed=5, tensor=0)
        ex, esx = ref.quantize(x.cpu().float().numpy())
        ew, esw = ref.quantize(W.cpu().float().numpy())
        ey, size = ref.linear(ex, esx, ew, esw, 0.25, 5, 0, None, ref.dbl(h))
        ref.check(y, ey, size, "bf16", 7)
        # the layer's end as two calls: product, then dropout and residual (one rounding more)
        plain = zgr.linear_i8(x, wq, ws)
        two = zgr.dropout(plain, 0.25, 5, 0, residual=h)
        ey2, size2 = ref.dropout(ref.dbl(plain), 0.25, 5, 0, None, ref.dbl(h))
        ref.check(two, ey2, size2, "bf16", 3)
        assert torch.equal(y == h, two == h)                            # the same elements are dropped
    z.restore_update(5, 2.0, 2.0, 0.1)


def test_streams_and_graphs():
    cases = []
    for m in (1, 8, 300):
        x, w = make((m, 500), "f16"), make((260, 500), "f16", 1)
        wq, ws = zgr.quantize_rows(w)
        cases.append((x, wq, ws, zgr.linear_i8(x, wq, ws, p=0.1, seed=1)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [zgr.linear_i8(x, wq, ws, p=0.1, seed=1, stream=side) for x, wq, ws, _ in cases]
    side.synchronize()
    for y, c in zip(got, cases):
        assert torch.equal(y, c[3])
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = [zgr.linear_i8(x, wq, ws, p=0.1, seed=1) for x, wq, ws, _ in cases]
        graphs.append((g, outs, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for g, _, s in graphs:
        with torch.cuda.stream(s):
            for _ in range(5):
                g.replay()
    torch.cuda.synchronize()
    for _, outs, _ in graphs:
        for y, c in zip(outs, cases):
            assert torch.equal(y, c[3])
    # new values in the same buffers are what a replay reads
    for x, *_ in cases:
        x.mul_(-1)
    graphs[0][0].replay()
    torch.cuda.synchronize()
    for y, (x, wq, ws, _) in zip(graphs[0][1], cases):
        assert torch.equal(y, zgr.linear_i8(x, wq, ws, p=0.1, seed=1))


def test_empty_batches_and_refusals():
    x, w = make((4, 64), "bf16"), make((24, 64), "bf16", 1)
    wq, ws = zgr.quantize_rows(w)
    assert zgr.linear_i8(x[:0], wq, ws).shape == (0, 24) and zgr.quantize_rows(x[:0])[0].shape == (0, 64)
    for bad in (lambda: zgr.linear_i8(x, wq[:, :32], ws), lambda: zgr.linear_i8(x, wq, ws[:3]), lambda: zgr.linear_i8(x, wq, None), lambda: zgr.linear_i8(x, w, ws),
                lambda: zgr.linear_i8(x.double(), wq, ws), lambda: zgr.linear_i8(x, wq, ws, bias=ws), lambda: zgr.linear_i8(x, wq, ws, residual=x),
                lambda: zgr.linear_i8(x.cpu(), wq, ws), lambda: zgr.linear_i8(x, wq.cpu(), ws), lambda: zgr.linear_i8(x, wq.t(), ws), lambda: zgr.quantize_rows(x, pitch=8),
                lambda: zgr.quantize_rows(x.view(-1)), lambda: zgr.matmul_i8(wq, ws, wq, ws, torch.float64), lambda: zgr.matmul_i8(x, ws, wq, ws)):
        with pytest.raises(ValueError):
            bad()
    odd = torch.zeros((24, 72), dtype=torch.int8, device="cuda")           # rows of codes off the 16-byte boundaries
    for bad in (lambda: zgr.linear_i8(x, odd[:, :64], ws), lambda: zgr.linear_i8(x, odd.view(-1)[8:8 + 24 * 64].view(24, 64), ws), lambda: zgr.linear_i8(x, wq, ws, p=1.5),
                lambda: zgr.matmul_i8(odd[:, :64], ws, wq, ws)):
        with pytest.raises(zgr.ZgrError) as e:
            bad()
        assert e.value.code == zgr.EINVAL


def test_a_chain_of_launches_sees_what_is_in_front_of_it():
    # weights requantised and tokens replaced between products whose launches overlap: the same as with a wait behind each.  The product
    # fetches weights before it waits for its tokens' quantiser; they may have been written by the call in front of that.
    def chain(m, wait):
        w, h = make((640, 640), "bf16", 1, 0.04), make((m, 640), "bf16", 2)
        for i in range(25):
            wq, ws = zgr.quantize_rows(w)
            if wait:
                torch.cuda.synchronize()
            h = zgr.linear_i8(h, wq, ws, residual=h, p=0.1, seed=i)
            if wait:
                torch.cuda.synchronize()
            zgr.dropout(w, 0.01, i, 7, out=w)
            h = h / h.float().std()
            h = h.bfloat16()
        return h
    for m in (1, 2, 9, 64, 700):
        assert torch.equal(chain(m, False), chain(m, True)), m


def test_rows_behind_each_other_at_large_offsets():
    # 2^32 results in front of the last rows: only a few rows of them are looked at
    k, n, m = 64, 70000, 62000
    x = make((128, k), "bf16").repeat((m + 127) // 128, 1)[:m]
    wq, ws = zgr.quantize_rows(make((n, k), "bf16", 1))
    y = zgr.linear_i8(x, wq, ws)
    assert y.numel() > 1 << 32
    small = zgr.linear_i8(x[:128], wq, ws)
    for row in (0, 30000, 61500, m - 1):
        assert torch.equal(y[row], small[row % 128])
    assert zgr.linear_status() == 0


def test_a_new_thread_may_begin_with_a_product_of_codes():
    # its first call of the driver is the description of the operands, which wants a context
    xq, xs = zgr.quantize_rows(make((48, 256), "bf16"))
    wq, ws = zgr.quantize_rows(make((200, 256), "bf16", 1))
    want, out, got = zgr.matmul_i8(xq, xs, wq, ws), torch.empty((48, 200), dtype=torch.bfloat16, device="cuda"), []
    torch.cuda.synchronize()

    def work():
        try:
            got.append(zgr.matmul_i8(xq, xs, wq, ws, out=out))
        except Exception as e:
            got.append(e)
    t = threading.Thread(target=work)
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert got[0] is out and torch.equal(out, want)


# tiles of 160 and 224 tokens by pairs, two CTAs on a multiprocessor, short inner dimensions with many tiles
@pytest.mark.parametrize("m,k,n", [(1000, 512, 11008), (4100, 512, 4096), (600, 300, 9000), (300, 4096, 4096), (333, 256, 20000), (5000, 64, 512)])
@pytest.mark.parametrize("residual", [False, True])
def test_whole_batches_and_parts_of_them_agree(m, k, n, residual):
    x, w = make((m, k), "bf16"), make((n, k), "bf16", 1)
    r = make((m, n), "bf16", 2) if residual else None
    (xq, xs), (wq, ws) = zgr.quantize_rows(x), zgr.quantize_rows(w)
    y = zgr.matmul_i8(xq, xs, wq, ws, residual=r)
    for at in range(0, m, 40):      # (another kernel and other tiles)
        assert torch.equal(zgr.matmul_i8(xq[at:at + 40], xs[at:at + 40], wq, ws, residual=None if r is None else r[at:at + 40]), y[at:at + 40]), at
    rows = [0, m // 2, m - 1]
    want = (xq[rows].double() @ wq.double().T) * xs[rows].double()[:, None] * ws.double() + (0 if r is None else r[rows].double())
    # the sum to fp32, the product of the scales, theirs and the residual: four roundings of 2^-24 of terms; the last of 2^-8
    size = want.abs() + (0 if r is None else 2 * r[rows].double().abs())
    assert bool(((y[rows].double() - want).abs() <= want.abs() * 2.0 ** -8 + size * 2.0 ** -21 + 1e-30).all())
    assert zgr.linear_status() == 0
