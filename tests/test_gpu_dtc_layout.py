"""Codes from quantize_rows as compressed coefficients: rows with a pitch are not what the sweeps read, and are refused."""
import pytest
import torch

from paper_2601_12917_b200 import zgr

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [200, 1000, 1024])
def test_rows_with_a_pitch_are_refused(cols):
    g = torch.Generator(device="cuda").manual_seed(1)
    G = torch.randn(16, cols, generator=g, device="cuda")
    U = torch.linalg.qr(torch.randn(96, 16, generator=g, device="cuda", dtype=torch.float64))[0].float().contiguous()
    w = torch.zeros(96, cols, device="cuda")
    z = zgr.Zgr([w], [U], 0.0, 1e-3)
    codes, scales = zgr.quantize_rows(G)                 # rows whole lines apart
    if cols % 128:
        assert not codes.is_contiguous()
        for call in (lambda: z.set_coeffs_dtc(0, codes, scales), lambda: z.set_coeffs_dtc_rows(0, codes, scales, None, 8, 16),
                     lambda: z.set_coeffs_dtc(0, codes.contiguous(), torch.stack([scales, scales], 1)[:, 0])):
            with pytest.raises(ValueError, match="contiguous"):
                call()
        codes = codes.contiguous()
    assert torch.equal(codes, zgr.quantize_rows(G, pitch=cols)[0])
    z.set_coeffs_dtc(0, codes, scales)
    z.perturb(9, 1.0)
    coefficients, b = codes.double() * scales.double()[:, None], z.scalars()[1]
    want, size = (U.double() @ coefficients) * b, (U.double().abs() @ coefficients.abs()) * b
    # fp32: the coefficient's product and its factor b, sixteen products and their sum, the addition to the weight: below 24 roundings of `size`
    assert bool(((w.double() - want).abs() <= 24 * 1.01 * 2.0 ** -24 * size).all())
