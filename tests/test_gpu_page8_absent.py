"""Selection of pages where the table lacks some of them, against the oracle, on the GPU: page numbers are equal."""
import numpy as np
import pytest
import torch

from oracle import page8_oracle as orc
from paper_2602_21780_b200 import binding
from tests.test_gpu_page8_ops import host, ints, made_up_pool

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,width,hkv", [(1, 70, 2), (3, 70, 8), (1, 2400, 1), (400, 90, 4), (300, 300, 8)])
@pytest.mark.parametrize("top,first,recent", [(9, 2, 3), (3, 1, 2), (5, 0, 5), (90, 40, 37)])
def test_pages_that_are_not_there_take_no_place_in_a_selection(tokens, width, hkv, top, first, recent):
    # a block a token, several blocks a token, several tokens a block; pages that the table lost anywhere, among the first and the last too
    d, pages = 64, 3000
    g = torch.Generator(device="cuda").manual_seed(width + top)
    pool, mean, factor = made_up_pool(pages, hkv, d, g)
    rng = np.random.default_rng(width + top)
    row = rng.permutation(pages)[:width].astype(np.int64)
    row[rng.random(width) < 0.3] = -1
    row[0], row[width - 2], row[rng.integers(1, width - 2)] = -1, -7, pages
    positions = [64 * width - 1] + [int(x) for x in rng.integers(0, 64 * width, tokens - 1)]
    q = torch.randn(tokens, 2 * hkv, d, device="cuda", generator=g).to(torch.bfloat16)
    sel = binding.page8_select(q, pool, ints(row[None]), ints([0] * tokens), ints(positions), top, first=first, recent=recent).cpu().numpy()
    there = [0 <= p < pages for p in row]
    for t in range(0, tokens, max(1, tokens // 40)):
        for h in range(hkv):
            means = [(mean[p, h], factor[p, h]) if 0 <= p < pages else None for p in row]
            want = orc.select(host(q[t, 2 * h:2 * h + 2]), means, positions[t] // 64, top, first, recent, there)
            assert sel[t, h].tolist() == want, (t, h)
    none = binding.page8_select(q, pool, ints(np.full((1, width), -1)), ints([0] * tokens), ints(positions), top, first=first, recent=recent)
    assert (none == -1).all()
