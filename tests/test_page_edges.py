"""Host side of the page operators where their descriptions end (no GPU needed)."""
import glob
import os

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_21780_b200", "csrc")


def test_kernels_read_memory_through_the_coherent_path():
    # Every kernel may be resident before the one that writes its inputs has ended; the read-only path (__ldg, ld.global.nc)
    # asks for data that nobody writes during the kernel's whole life.
    for path in glob.glob(os.path.join(CSRC, "*.cu*")):
        src = open(path).read()
        assert "__ldg(" not in src and "ld.global.nc" not in src, path
