"""Appends of prompts to 8-bit pages by blocks that take several heads, on the GPU: codes, scales and mean keys are those of the oracle."""
import numpy as np
import pytest

from tests.test_gpu_page8_ops import Server

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d,hkv,n", [(64, 8, 9700), (128, 8, 9700), (128, 5, 9600), (64, 7, 4900), (128, 3, 9500)])
def test_append_of_prompts_by_blocks_that_take_several_heads(dtype, d, hkv, n):
    # So many tokens that a block stores up to four heads of a page one after the other, the last block fewer.  Prompts begin in
    # pages that hold tokens already, whose codes move to a larger scale, end anywhere, and some tokens come one at a time.
    sv = Server(6, hkv, d, dtype, pages=200, width=100, seed=d + hkv)
    sv.step([0, 7, 40, 63, 128, 250], sizes=[0.1] * 488)
    a, b = n // 3 + 5, n // 2 - 3
    new = [a, b, n - a - b - 52, 1, 31, 20]
    sv.step(new, pad=5, sizes=np.exp2(np.random.default_rng(n).integers(-3, 4, n)).tolist() + [0.0] * 5)
    sv.check_state()
