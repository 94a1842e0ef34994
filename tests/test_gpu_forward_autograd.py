"""Autograd and the operators of the forward pass: they record nothing, so what would lose a gradient or keep a stale history is refused."""
import pytest
import torch

from paper_2601_12917_b200 import zgr

pytestmark = pytest.mark.gpu


def given():
    g = torch.Generator(device="cuda").manual_seed(2)
    t = lambda *s: torch.randn(*s, generator=g, device="cuda")
    wq, ws = zgr.quantize_rows(t(24, 64))
    xq, xs = zgr.quantize_rows(t(12, 64))
    return dict(x=t(12, 64), bias=t(64), residual=t(12, 64), out=t(12, 64), wq=wq, ws=ws, xq=xq, xs=xs, b=t(24), r=t(12, 24), o=t(12, 24))


CALLS = {
    "dropout": (lambda v: zgr.dropout(v["x"], 0.5, 1, bias=v["bias"], residual=v["residual"], out=v["out"]), ("x", "bias", "residual", "out")),
    "dropout_backward": (lambda v: zgr.dropout_backward(v["x"], 0.5, 1, out=v["out"]), ("x", "out")),
    "dropout_backward_bias": (lambda v: zgr.dropout_backward(v["x"], 0.5, 1, bias_grad=True, out=v["out"])[0], ("x", "out")),
    "linear_i8": (lambda v: zgr.linear_i8(v["x"], v["wq"], v["ws"], bias=v["b"], residual=v["r"], out=v["o"]), ("x", "ws", "b", "r", "o")),
    "matmul_i8": (lambda v: zgr.matmul_i8(v["xq"], v["xs"], v["wq"], v["ws"], torch.float32, bias=v["b"], residual=v["r"], out=v["o"]), ("xs", "ws", "b", "r", "o")),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_what_requires_gradients_is_refused_while_they_are_recorded(name):
    call, places = CALLS[name]
    want = call(given()).clone()
    for place in places:
        v = given()
        v[place].requires_grad_()
        before = {k: t.detach().clone() for k, t in v.items()}
        with pytest.raises(ValueError, match="requires gradients"):
            call(v)
        assert all(torch.equal(v[k], t) for k, t in before.items())         # nothing was written
        with torch.no_grad():
            assert torch.equal(call(v), want)
        v[place].requires_grad_(False)
        assert torch.equal(call(given()), want)
    # a result of recorded work, which is no leaf
    v = given()
    v[places[0]] = (v[places[0]].requires_grad_() * 1.0)
    with pytest.raises(ValueError, match="requires gradients"):
        call(v)
    v = given()
    for place in places:
        v[place].requires_grad_()
    with torch.inference_mode():
        assert torch.equal(call({k: t.clone() for k, t in v.items()}), want)


def test_parameters_are_quantised_as_they_are():
    w = torch.nn.Parameter(torch.randn(24, 64, device="cuda"))
    codes, scales = zgr.quantize_rows(w)
    with torch.no_grad():
        again, scales2 = zgr.quantize_rows(w)
    assert torch.equal(codes, again) and torch.equal(scales, scales2) and not scales.requires_grad
