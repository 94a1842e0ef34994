"""Cases of the forward-pass operators: dropout from the counter-based generator (forward, backward) and the 8-bit matrix product
with a scale for each token and each channel, alone and behind the requantisation of its weights.

Sizes are those of the parameter sets of this repository (RoBERTa-large 1024/4096/50265, OPT-1.3B 2048/8192, LLaMA-7B
4096/11008, LLaMA-13B 5120/13824), batches of single tokens up to 8 sequences of 1024, and odd ones between them.

Every operator has a plain form in elementary torch operations (``own`` false) and the library's call (``own`` true).
"""
import functools
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
TENSOR = 5             # generator's tensor id of the masked activation
TAG = 2                # generator's stream tag of dropout
TINY = 2.0 ** -120     # a row whose largest magnitude is below this counts as zero


# ------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token's hidden state between two layers while a sequence is generated
        dict(name="dropout_one_token", op="dropout", dtype="bf16", rows=1, cols=4096, p=0.1, bias=True, residual=True),
        # eight sequences of 1024 tokens, LLaMA-7B width, end of a block: dropout and the residual's sum
        dict(name="dropout_batch", op="dropout", dtype="bf16", rows=8192, cols=4096, p=0.1, bias=False, residual=True),
        # attention probabilities of 16 heads over a context that is not a multiple of anything
        dict(name="dropout_odd", op="dropout", dtype="f16", rows=16 * 1021, cols=1021, p=0.25, bias=False, residual=False),
        # the cloud's back-propagation: OPT-1.3B width with the bias's gradient, RoBERTa-large width in fp32
        dict(name="dropout_backward_bias", op="backward", dtype="f16", rows=8192, cols=2048, p=0.1, bias=True),
        dict(name="dropout_backward_f32", op="backward", dtype="f32", rows=4096, cols=1024, p=0.5, bias=False),
        # single token into the gated FFN; a small batch of tokens out of it; a batch of 64 at LLaMA-13B sizes
        dict(name="linear_one_token", op="linear", dtype="bf16", m=1, k=4096, n=11008, p=0.0, bias=False, residual=False),
        dict(name="linear_eight_tokens", op="linear", dtype="bf16", m=8, k=11008, n=4096, p=0.0, bias=False, residual=True),
        dict(name="linear_batch64", op="linear", dtype="bf16", m=64, k=5120, n=13824, p=0.0, bias=False, residual=False),
        # eight sequences of 1024 tokens
        dict(name="linear_prefill", op="linear", dtype="bf16", m=8192, k=4096, n=11008, p=0.0, bias=False, residual=False),
        # RoBERTa-large's vocabulary (odd), a ragged batch, an inner size that is no multiple of 16, fp32
        dict(name="linear_odd_f32", op="linear", dtype="f32", m=333, k=1027, n=50265, p=0.0, bias=True, residual=False),
        # after a sweep over the weights: OPT-1.3B's FFN requantised and applied, with the block's dropout and residual
        dict(name="requantised_block_end", op="requantised", dtype="f16", m=1024, k=8192, n=2048, p=0.1, bias=True, residual=True),
        dict(name="requantised_one_token", op="requantised", dtype="bf16", m=1, k=4096, n=4096, p=0.0, bias=False, residual=False),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return min(max(v, lo), hi)


def _size(rng, lo, hi):
    """A size, spread over the logarithm; half of them whole multiples of 64, as widths of models are."""
    v = _log(rng, lo, hi)
    return max(64, v // 64 * 64) if v >= 64 and rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(["dropout", "backward", "linear", "linear", "requantised"])
    c = dict(op=op, dtype=rng.choice(["f32", "f16", "bf16", "bf16"]), p=rng.choice([0.0, 0.1, 0.25, 0.5]), bias=rng.random() < 0.5)
    if op in ("dropout", "backward"):
        c["p"] = round(rng.uniform(0.02, 0.9), 3)
        c["rows"], c["cols"] = _log(rng, 1, 16384), _size(rng, 1, 16384)
        if c["rows"] * c["cols"] * SIZE[c["dtype"]] > 1 << 26:
            c["rows"] = max(1, (1 << 26) // (c["cols"] * SIZE[c["dtype"]]))
    else:
        c["m"], c["k"], c["n"] = _log(rng, 1, 8192), _size(rng, 16, 13824), _size(rng, 16, 32000)
        if op == "requantised" and c["n"] * c["k"] > 1 << 26:
            c["n"] = (1 << 26) // c["k"]
        if c["m"] * c["n"] * c["k"] > 1 << 38:
            c["m"] = max(1, (1 << 38) // (c["n"] * c["k"]))
    if op != "backward":
        c["residual"] = rng.random() < 0.5
    return c


# ------------------------------------------------------------------------------------------------------------ inputs
def _quantised(x):
    """Codes and scales of the rows of x, by the definition: with a the largest magnitude, scale fl(a / 127), code
    rint(fl(x fl(127 / a)))."""
    x = x.float()
    a = x.abs().amax(dim=1, keepdim=True)
    some = a >= TINY
    inv = torch.where(some, 127.0 / a, torch.zeros_like(a))
    codes = (x * inv).round().clamp(-127, 127)
    return codes, torch.where(some, a / 127.0, torch.zeros_like(a))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(shape, sigma):
        return (torch.randn(shape, generator=g, device="cuda") * sigma).to(dt)

    st = {"case": case, "mask_seed": (seed * 2654435761 + 97) & 0xFFFFFFFFFFFFFFFF}
    if case["op"] in ("dropout", "backward"):
        rows, cols = case["rows"], case["cols"]
    else:
        rows, cols = case["m"], case["n"]
    if case["op"] == "dropout":
        st["x"] = normal((rows, cols), 1.0)
    elif case["op"] == "backward":
        st["dy"] = normal((rows, cols), 0.1)
    else:
        # hidden states: unit normals with a few channels several times as large
        x = torch.randn((case["m"], case["k"]), generator=g, device="cuda")
        x[:, :: 97] *= 4.0
        st["x"] = x.to(dt)
        w = normal((case["n"], case["k"]), 0.02)
        if case["op"] == "requantised":
            st["w"] = w
        else:
            # rows of codes start on 16-byte boundaries, as the library's quantiser lays them out
            codes, scale = _quantised(w)
            held = torch.zeros((case["n"], (case["k"] + 15) // 16 * 16), dtype=torch.int8, device="cuda")
            held[:, : case["k"]] = codes.to(torch.int8)
            st["wq"], st["ws"] = held[:, : case["k"]], scale.reshape(-1).contiguous()
    st["bias"] = normal((cols,), 0.1) if case["bias"] and case["op"] != "backward" else None
    st["residual"] = normal((rows, cols), 1.0) if case.get("residual") else None
    return st


# ------------------------------------------------------------------------------------------------------- plain forms
def _round(words, key):
    c0, c1, c2, c3 = words
    p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57          # 64-bit products; the high half is masked after the shift
    low = 0xFFFFFFFF
    return ((p1 >> 32) & low) ^ c1 ^ key[0], p1 & low, ((p0 >> 32) & low) ^ c3 ^ key[1], p0 & low


def _keep(rows, cols, p, seed, device):
    """Truth values, rows x cols: which elements the mask of (seed, TENSOR) keeps."""
    per_row = (cols + 7) // 8
    block = torch.arange(rows * per_row, dtype=torch.int64, device=device)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    keys = [((k0 + r * 0x9E3779B9) & 0xFFFFFFFF, (k1 + r * 0xBB67AE85) & 0xFFFFFFFF) for r in range(10)]
    zero = torch.zeros_like(block)
    words = functools.reduce(_round, keys, (block & 0xFFFFFFFF, block >> 32, zero + TENSOR, zero + TAG))
    words = torch.stack(words, dim=1)
    halves = torch.stack((words & 0xFFFF, words >> 16), dim=2).reshape(rows, per_row * 8)
    return halves[:, :cols] >= round(65536 * p)


def _factor(p):
    t = round(65536 * p)
    return 65536.0 / (65536 - t) if t < 65536 else 0.0


def _masked(v, p, seed):
    keep = _keep(v.shape[0], v.shape[1], p, seed, v.device)
    return torch.where(keep, v * _factor(p), torch.zeros_like(v))


def _plain(st):
    case, p, seed = st["case"], st["case"]["p"], st["mask_seed"]
    dt = DTYPES[case["dtype"]]
    if case["op"] == "backward":
        dx = _masked(st["dy"].float(), p, seed)
        return (dx.to(dt), dx.sum(dim=0).to(dt)) if case["bias"] else dx.to(dt)
    if case["op"] == "dropout":
        y = st["x"].float()
    else:
        qw, ws = _quantised(st["w"]) if case["op"] == "requantised" else (st["wq"].float(), st["ws"])
        qx, xs = _quantised(st["x"])
        y = (qx @ qw.t()) * (xs.reshape(-1, 1) * ws.reshape(1, -1))
    if st["bias"] is not None:
        y = y + st["bias"].float()
    if case["op"] == "dropout" or p > 0:
        y = _masked(y, p, seed)
    if st["residual"] is not None:
        y = st["residual"].float() + y
    return y.to(dt)


def run(state):
    if not own:
        return _plain(state)
    from paper_2601_12917_b200 import zgr
    case = state["case"]
    if case["op"] == "backward":
        return zgr.dropout_backward(state["dy"], case["p"], state["mask_seed"], TENSOR, bias_grad=case["bias"])
    if case["op"] == "dropout":
        return zgr.dropout(state["x"], case["p"], state["mask_seed"], TENSOR, bias=state["bias"], residual=state["residual"])
    wq, ws = zgr.quantize_rows(state["w"]) if case["op"] == "requantised" else (state["wq"], state["ws"])
    return zgr.linear_i8(state["x"], wq, ws, bias=state["bias"], residual=state["residual"], p=case["p"], seed=state["mask_seed"],
                         tensor=TENSOR)


# -------------------------------------------------------------------------------------------------------------- work
def work(case):
    size = SIZE[case["dtype"]]
    if case["op"] in ("dropout", "backward"):
        n = case["rows"] * case["cols"]
        extra = (case["cols"] if case["bias"] else 0) + (n if case.get("residual") else 0)
        return {"bytes": (2 * n + extra) * size, "flops": 2 * n}
    m, k, n = case["m"], case["k"], case["n"]
    weights = n * k * size if case["op"] == "requantised" else n * k + 4 * n
    extra = (n if case["bias"] else 0) + (m * n if case["residual"] else 0)
    return {"bytes": m * k * size + weights + (m * n + extra) * size, "flops": 2 * m * n * k}


# ------------------------------------------------------------------------------------------- definitions in 64 bits
def _exact_keep(rows, cols, p, seed):
    """The mask from the generator's definition, in numpy's unsigned integers."""
    per_row = -(-cols // 8)
    j = np.arange(rows * per_row, dtype=np.uint64)
    low, s32 = np.uint64(0xFFFFFFFF), np.uint64(32)
    x = [j & low, j >> s32, np.full_like(j, TENSOR), np.full_like(j, TAG)]
    key = [seed % (1 << 32), seed >> 32]
    for _ in range(10):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> s32) ^ x[1] ^ np.uint64(key[0]), b & low, (a >> s32) ^ x[3] ^ np.uint64(key[1]), a & low]
        key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
    half = np.empty((rows * per_row, 8), dtype=np.uint32)
    for w in range(4):
        half[:, 2 * w] = x[w] & np.uint64(0xFFFF)
        half[:, 2 * w + 1] = x[w] >> np.uint64(16)
    return half.reshape(rows, per_row * 8)[:, :cols] >= int(np.rint(65536.0 * p))


def _exact_codes(x):
    """Codes (whole numbers, in 64 bits) and scales.  The scale, its reciprocal and the product that is rounded to a code are fp32
    numbers by definition, so that a code next to a border is the same everywhere."""
    x = x.cpu().float().numpy()
    a = np.abs(x).max(axis=1, keepdims=True)
    zero = a < TINY
    safe = np.where(zero, np.float32(1), a).astype(np.float32)
    codes = np.rint(x * (np.float32(127) / safe)).clip(-127, 127)
    codes[zero[:, 0]] = 0
    return torch.from_numpy(codes.astype(np.float64)), torch.from_numpy(np.where(zero, 0.0, (safe / np.float32(127)).astype(np.float64)))


def exact(case, seed):
    st = prepare(case, seed)
    p = case["p"]
    t = int(np.rint(65536.0 * p))
    gain = 65536.0 / (65536 - t) if t < 65536 else 0.0
    if case["op"] == "backward":
        v = st["dy"].double().cpu()
    elif case["op"] == "dropout":
        v = st["x"].double().cpu()
    else:
        qx, sx = _exact_codes(st["x"])
        if case["op"] == "requantised":
            qw, sw = _exact_codes(st["w"])
        else:
            qw, sw = st["wq"].cpu().double(), st["ws"].cpu().double().reshape(-1, 1)
        v = torch.mm(qx.cuda(), qw.cuda().t()).cpu() * sx * sw.t()
    if st["bias"] is not None:
        v = v + st["bias"].double().cpu()
    if case["op"] in ("dropout", "backward") or p > 0:
        keep = torch.from_numpy(_exact_keep(v.shape[0], v.shape[1], p, st["mask_seed"]))
        v = torch.where(keep, v * gain, torch.zeros_like(v))
    if case["op"] == "backward":
        return (v, v.sum(dim=0)) if case["bias"] else v
    if st["residual"] is not None:
        v = v + st["residual"].double().cpu()
    return v
