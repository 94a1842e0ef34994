"""Codes next to a border between two of them: the kernel against its definition, and both against the nearest integer of x * 127 / a.

The definition takes products with fp32 reciprocals.  With u = 2^-24: 1/a is off by u, its product with 127 by another, the product with x by a third, so
the number that is rounded to a code differs from x * 127 / a by at most 3.01 u of it, of at most 127: a code may be the other neighbour only
within 127 * 3.01 u of a border.  A form with quotients (127 / a, then the product) is off by two such roundings, within the same bound."""
import numpy as np
import pytest
import torch

import forward_ref as ref
import oracle
from paper_2601_12917_b200 import zgr

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
NEAR = 127 * 3.01 * U


def distance(t):
    """Of t from the border between two codes that is nearest to it."""
    return np.abs(t - np.floor(t) - 0.5)


def halves(dtype):
    """Rows of which many elements lie on or next to borders: (j + 1/2) / 127 of the largest magnitude a and the numbers beside it."""
    rows = []
    g = np.random.default_rng(3)
    for a in [127.0, 254.0, 63.5, 1.0, 0.75, 100.0, 2.0 ** -10, 3.0, 127 * 2.0 ** -12] + list(np.exp(g.uniform(-8, 8, 23))):
        top = torch.tensor(a, dtype=ref.DTYPES[dtype]).double().item()
        at = top * (np.arange(-127, 127) + 0.5) / 127
        x = torch.from_numpy(np.concatenate([[top], at, at / 2, [top / 2, -top / 2, -top]])).to(ref.DTYPES[dtype])
        up, down = torch.nextafter(x, torch.full_like(x, float("inf"))), torch.nextafter(x, torch.full_like(x, float("-inf")))
        both = torch.stack([x, up, down])
        rows.append(torch.where(both.double().abs() > top, x, both).reshape(-1))      # (nothing above the largest magnitude)
    return torch.stack(rows)


@pytest.mark.parametrize("dtype", list(ref.DTYPES))
def test_codes_next_to_borders(dtype):
    x = halves(dtype)
    x = torch.cat([x, torch.randn(40, x.shape[1], generator=torch.Generator().manual_seed(4)).to(x.dtype)])
    codes, scales = zgr.quantize_rows(x.cuda())
    ec, es = ref.quantize(x.float().numpy())
    assert np.array_equal(codes.cpu().numpy().astype(np.int64), ec) and np.array_equal(scales.cpu().numpy(), es)
    d = x.double().numpy()
    a = np.abs(d).max(axis=1, keepdims=True)
    t = d * 127 / a
    q = np.rint(x.float().numpy() * (np.float32(127) / a.astype(np.float32))).astype(np.int64)      # with a quotient
    for c in (ec, q):
        other = c != np.rint(t)
        assert np.abs(c - t).max() <= 0.5 + NEAR and (distance(t)[other] <= NEAR).all()
    assert (distance(t) < NEAR).any() and (np.abs(es.astype(np.float64) / (a[:, 0] / 127) - 1) <= 2.01 * U).all()


def test_codes_of_the_oracle_but_next_to_borders():
    # the compressed coefficients' codes: the oracle divides by its scale, off by u of a / 127
    G = torch.randn(300, 1000, generator=torch.Generator().manual_seed(9))
    codes, scales = zgr.quantize_rows(G.cuda(), pitch=1000)
    eq, es, _ = oracle.dtc_quantise(G.double().numpy(), 8, True)
    es = np.asarray(es, dtype=np.float64).reshape(-1, 1)
    other = codes.cpu().numpy().astype(np.int64) != np.asarray(eq).reshape(300, 1000)
    assert (distance(G.double().numpy() / es)[other] <= NEAR + 127 * 1.01 * U).all() and other.mean() < 1e-4
