"""Which kernel serves a product of which size (zgr_debug_linear_plan), and that the sizes of the GPU tests reach every form; no device."""
import ctypes
import random

import pytest

import test_gpu_linear_forms as forms
from paper_2601_12917_b200 import zgr


@pytest.mark.parametrize("bad", [(0, 8, 8), (-1, 8, 8), (4, 0, 8), (4, 8, 0), (4, 8, (1 << 17) + 1), (1 << 31, 8, 8), (4, 1 << 31, 8)])
def test_sizes_that_the_products_refuse(bad):
    for codes in (0, 1):
        assert zgr.lib().zgr_debug_linear_plan(*bad, codes, ctypes.byref(zgr.LinearPlan())) == zgr.EINVAL
    assert zgr.lib().zgr_debug_linear_plan(4, 8, 8, 0, None) == zgr.EINVAL


def test_plans_are_what_the_kernels_can_do():
    rng = random.Random(5)
    for _ in range(4000):
        m, n, k = (int(2 ** rng.uniform(0, top)) for top in (14, 17, 17))
        kernel, tokens, split = zgr.debug_linear_plan(m, n, k)
        # the tokens' codes need a workspace unless the product makes them itself
        assert (kernel == zgr.LINEAR_FEW) == (zgr.lib().zgr_linear_i8_workspace(m, n, k) == 0)
        if kernel == zgr.LINEAR_FEW:
            assert tokens == m <= 8 and split == 1
            kernel, tokens, split = zgr.debug_linear_plan(m, n, k, codes=True)
        assert kernel in (zgr.LINEAR_TILE, zgr.LINEAR_PAIR) and tokens % (32 if kernel == zgr.LINEAR_PAIR else 16) == 0 and 16 <= tokens <= 256
        assert split in ((1,) if kernel == zgr.LINEAR_PAIR else (1, 2, 4)) and (split == 1 or -(-k // 128) >= 2 * split)
        if m > 8:
            assert (kernel, tokens, split) == zgr.debug_linear_plan(m, n, k, codes=True)


def test_the_gpu_tests_sizes_reach_every_form():
    for m, k, n, plan in forms.PAIRS + forms.PAIRS_MORE + forms.SPLIT:
        assert zgr.debug_linear_plan(m, n, k) == plan, (m, k, n)
    assert {p[1] for *_, p in forms.PAIRS + forms.PAIRS_MORE} >= {96, 128, 160, 192, 224, 256}
    assert {p[2] for *_, p in forms.SPLIT} == {2, 4}
    m, k, n, parts = forms.SAME_BITS
    assert zgr.debug_linear_plan(m, n, k)[0] == zgr.LINEAR_PAIR
    assert {zgr.debug_linear_plan(mm, nn, k)[::2] for mm, nn in parts} == {(zgr.LINEAR_FEW, 1), (zgr.LINEAR_TILE, 1), (zgr.LINEAR_TILE, 2), (zgr.LINEAR_TILE, 4)}
