"""The operators over a shared pool of 4-bit pages where their descriptions end: hand-overs between the kernels' roles, the
ends of the number range, refused sequences, bounds that are too small, scales that underflow."""
import numpy as np
import pytest
import torch

from oracle import page_oracle as orc
from paper_2602_21780_b200 import binding
from tests.test_gpu_page_ops import DT, HALF, PAGE, Server, host, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,hq,hkv,new", [(64, 3, 3, 101), (128, 4, 2, 60)])
def test_long_units_without_a_second_query_tile(d, hq, hkv, new):
    # at most 128 query rows a head over more pages than the ring of stages holds twice: the warp that would serve the second
    # tile passes every stage's phases and releases its share of them; a longer chunk beside it changes between both kinds
    sv = Server(3, hkv, d, "bf16", pages=170, width=64, seed=d + new)
    sv.step([3003, 2500, 1100])
    for step in ([new, 0, 0], [new, 400, new + 1], [0, new, 300]):
        plan = sv.step(step)
        sv.check_attention(plan, step, hq)
