"""Host side of the page operators where their descriptions end (no GPU needed)."""
import glob
import os

import numpy as np

from oracle import page_oracle as orc
from paper_2602_21780_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_21780_b200", "csrc")


def test_kernels_read_memory_through_the_coherent_path():
    # Every kernel may be resident before the one that writes its inputs has ended; the read-only path (__ldg, ld.global.nc)
    # asks for data that nobody writes during the kernel's whole life.
    for path in glob.glob(os.path.join(CSRC, "*.cu*")):
        src = open(path).read()
        assert "__ldg(" not in src and "ld.global.nc" not in src, path


def test_no_code_stands_for_more_than_the_largest_half():
    rng = np.random.default_rng(5)
    top, ulp = 65504.0, 32.0
    x = [np.r_[lo, top, rng.uniform(lo, top, 62)] for lo in (0.0, -65504.0, -60000.0, 65472.0, 65000.0, 1e-7, -1e-7, 40000.0)]
    x += [np.r_[-top, rng.uniform(-top, 60000, 63)], np.full(64, top), np.full(64, -top), np.r_[top - ulp * np.arange(64)]]
    x = np.stack(x + [np.r_[lo, rng.uniform(lo, top, 63)].astype(np.float16).astype(np.float64) for lo in rng.uniform(-top, top, 300)])
    c, s, z = orc.quantise(x, 1)
    assert c.min() >= 0 and c.max() <= 15
    value = c * s + z
    assert np.all(np.abs(value) <= top) and np.all(np.isfinite(value.astype(np.float16)))
    assert np.all((15 * s + z)[s[:, 0] != 1] <= top)
    assert np.all(np.abs(value - x) <= s / 2 * (1 + 1e-12))


def test_plan_refuses_rows_of_more_tokens_than_32_bits_count():
    a = 1 << 20
    args = [a, a + 64, 2, a, (1 << 24) + 1, a, 9, a, a + 64, a + 128, a + 256, a, a, a, 5, None]
    assert binding.load().xsv_page_plan(*args) == 9
