"""The forward-pass operators on a stream of their own: memory that the caller lets go of stays theirs until that stream is done with it."""
import pytest
import torch

from paper_2601_12917_b200 import zgr

pytestmark = pytest.mark.gpu
DELAY = 400_000_000      # cycles, some 0.2 s: longer than a busy host takes between two calls


def normal(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def calls():
    w, ws = zgr.quantize_rows(normal(512, 640, seed=9))
    def matmul(x, r, s):
        q, qs = zgr.quantize_rows(x)
        if s is not None:
            s.wait_stream(torch.cuda.current_stream())      # the codes are made on the current stream
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                torch.cuda._sleep(DELAY)
        return zgr.matmul_i8(q, qs, w, ws, torch.float32, residual=r[:, :512], stream=s)
    return {"dropout": lambda x, r, s: zgr.dropout(x, 0.5, 1, residual=r, bias=x[0].clone(), stream=s),
            "dropout_backward": lambda x, r, s: zgr.dropout_backward(x, 0.5, 1, bias_grad=True, stream=s)[0],
            "quantize_rows": lambda x, r, s: zgr.quantize_rows(x, stream=s)[0],
            "linear_i8": lambda x, r, s: zgr.linear_i8(x, w, ws, residual=r[:, :512], stream=s),
            "matmul_i8": matmul}


@pytest.mark.parametrize("name", ["dropout", "dropout_backward", "quantize_rows", "linear_i8", "matmul_i8"])
def test_inputs_that_are_let_go_of(name):
    call = calls()[name]
    want = call(normal(700, 640), normal(700, 640, seed=1), None).clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(DELAY)
    x, r = normal(700, 640), normal(700, 640, seed=1)
    torch.cuda.current_stream().synchronize()           # (the inputs are there; what follows only has to outlive the delay)
    got = call(x, r, side)
    assert not side.query(), "the delay was too short to show anything"
    del x, r
    # the next owners of whatever memory was let go of write into it at once
    others = [torch.full((n,), 7e4, device="cuda") for n in 6 * (700 * 640, 640, 700, 700 * 160)]
    torch.cuda.current_stream().synchronize()
    side.synchronize()
    assert torch.equal(got, want)
    del others


def test_results_that_are_let_go_of():
    # a result made on the side stream and read on the current one: its memory is not the side stream's again before that read
    side = torch.cuda.Stream()
    x = normal(700, 640)
    want = zgr.dropout(x, 0.5, 1).clone()
    torch.cuda.synchronize()
    y = zgr.dropout(x, 0.5, 1, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(DELAY)
    copy = y.clone()
    del y
    others = [zgr.dropout(x, 0.5, i, stream=side) for i in range(2, 6)]
    side.synchronize()
    assert not torch.cuda.current_stream().query(), "the delay was too short to show anything"
    torch.cuda.synchronize()
    assert torch.equal(copy, want)
    del others


def test_a_forked_stream_in_a_graph():
    w, ws = zgr.quantize_rows(normal(512, 640, seed=9))
    x, r = normal(700, 640), normal(700, 512, seed=1)

    def work(side):
        side.wait_stream(torch.cuda.current_stream())
        a = zgr.linear_i8(x * 2, w, ws, residual=r, stream=side)
        b = zgr.linear_i8(x, w, ws)
        torch.cuda.current_stream().wait_stream(side)
        return a + b, zgr.dropout(a, 0.3, 4, residual=b)
    want = [t.clone() for t in work(torch.cuda.Stream())]
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = work(torch.cuda.Stream())
        graphs.append((g, out))
    for _ in range(3):
        for g, out in graphs:
            for t in out:
                t.zero_()
            g.replay()
            assert all(torch.equal(a, b) for a, b in zip(out, want))
    for _ in range(3):                                   # and eager work afterwards, on what the graphs do not own
        assert all(torch.equal(a, b) for a, b in zip(work(torch.cuda.Stream()), want))
