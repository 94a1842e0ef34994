"""What a product leaves behind when one of its bounded waits runs out: no wrong results, a status that says so, and a device that works on.

The first wait of one thread block counts as run out (zgr_debug_matmul_i8_giving_up): that block fetches nothing, and all that would have waited for it
gives up too.  In a process of its own, because the status word stays set."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = """
import sys
import torch
sys.path.insert(0, sys.argv[1])
from paper_2601_12917_b200 import zgr

kernel, tokens, split = (int(a) for a in sys.argv[2].split(","))
m, k, n = (int(a) for a in sys.argv[3].split(","))
block, residual = int(sys.argv[4]), int(sys.argv[5])
assert zgr.debug_linear_plan(m, n, k, codes=True) == (kernel, tokens, split), zgr.debug_linear_plan(m, n, k, codes=True)
g = torch.Generator(device="cuda").manual_seed(1)
x, w = (torch.randn(s, generator=g, device="cuda") for s in ((m, k), (n, k)))
r = torch.randn((m, n), generator=g, device="cuda") if residual else None
(xq, xs), (wq, ws) = zgr.quantize_rows(x), zgr.quantize_rows(w)
good = zgr.matmul_i8(xq, xs, wq, ws, torch.float32, residual=r, p=0.1, seed=3)
assert zgr.linear_status() == 0

# the elements of the tiles that this block has a part in
token_tiles = -(-m // tokens)
lost = torch.zeros((m, n), dtype=torch.bool, device="cuda")
if kernel == zgr.LINEAR_TILE:
    tiles, channels = [block // split], 128
else:
    count = -(-n // 256) * token_tiles
    tiles, channels = range(block // 2, count, min(count, 74)), 256
for t in tiles:
    lost[t % token_tiles * tokens:][:tokens, t // token_tiles * channels:][:, :channels] = True
assert bool(lost.any()) and not bool(lost.all())

y = torch.full((m, n), 77.0, device="cuda")
rc = zgr.lib().zgr_debug_matmul_i8_giving_up(xq.data_ptr(), xq.stride(0), xs.data_ptr(), wq.data_ptr(), wq.stride(0), ws.data_ptr(), None, r.data_ptr() if residual else None, n,
                                             y.data_ptr(), n, m, n, k, zgr.F32, 0.1, 3, 0, block, torch.cuda.current_stream().cuda_stream)
assert rc == zgr.OK
assert zgr.linear_status() == 100
assert bool((y[lost] == 77.0).all()), "results without their sums"
assert torch.equal(y[~lost], good[~lost])
assert torch.equal(zgr.matmul_i8(xq, xs, wq, ws, torch.float32, residual=r, p=0.1, seed=3), good)
assert zgr.linear_status() == 100
print("as documented")
"""


# kernel, tokens of a tile, CTAs of a tile; m, k, n; the block
@pytest.mark.parametrize("plan,size,block", [("1,32,1", "60,2050,5000", 5), ("1,16,2", "17,1500,140", 2), ("1,16,2", "17,1500,140", 3), ("1,48,4", "70,4100,2000", 4),
                                             ("1,48,4", "70,4100,2000", 7), ("2,96,1", "257,17,20001", 0), ("2,96,1", "257,17,20001", 13), ("2,128,1", "200,1100,20001", 8),
                                             ("2,128,1", "200,1100,20001", 1)])
@pytest.mark.parametrize("residual", [0, 1])
def test_a_wait_that_runs_out(plan, size, block, residual):
    r = subprocess.run([sys.executable, "-c", CHILD, ROOT, plan, size, str(block), str(residual)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "as documented" in r.stdout, r.stdout + r.stderr
