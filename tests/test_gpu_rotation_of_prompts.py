"""Norm and rotation of so many tokens that a block has two of them in flight, or may have, against the float64 oracle, on the GPU.  Tolerances are those of
test_gpu_page_ops.py: half a step of the output type and 2e-5 of a row's largest element."""
import numpy as np
import pytest
import torch

from oracle import page8_oracle as orc8
from oracle import page_oracle as orc
from paper_2602_21780_b200 import binding
from tests.test_gpu_page_ops import DT, HALF, host, ints

pytestmark = pytest.mark.gpu

# on 148 multiprocessors, a turn of two tokens a block is 2072: one that is a fifth over, two within the second, just beyond two, the fourth
COUNTS = [2489, 3500, 4145, 8191]


def check(dtype, d, hq, hkv, n, norm, rope, rotary, several):
    dt, r = DT[dtype], rotary or d
    g = torch.Generator(device="cuda").manual_seed(d + n)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    fused = (rnd(n, (hq + 2 * hkv) * d + 8) * (0.1 + 3 * torch.rand(n, 1, device="cuda", generator=g)) + 0.3).to(dt)
    q, k, v = (fused[:, a * d:b * d].view(n, b - a, d) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
    w = [(1 + 0.3 * rnd(d)).to(dt), None, (1 + 0.3 * rnd(d)).to(dt), (0.2 * rnd(d)).to(dt)] if norm else [None] * 4
    rng, kw = np.random.default_rng(n), {}
    inv = pos = axes = None
    if rope == "2d":
        inv, pos = 100.0 ** (-torch.arange(d // 4, device="cuda") / (d / 4)), rng.integers(0, 40, (n, 2))
    elif rope:
        inv = 10000.0 ** (-torch.arange(r // 2, device="cuda") / (r / 2))
        pos = rng.integers(-5, 2_000_000, (n, several) if several else n)
    if several:
        axes = rng.integers(0, several, r // 2)
        axes[rng.integers(0, r // 2, 2)] = (-1, several)         # no such position: not rotated
        kw["axes"] = ints(axes)
    if rope:
        kw.update(rope=rope, inv_freq=inv, positions=ints(pos))
    kw.update(norm=norm, q_weight=w[0], q_bias=w[1], k_weight=w[2], k_bias=w[3], eps=1e-5)
    out = binding.qk_norm_rope(q, k, v, **kw)
    assert torch.equal(out[2], v)
    for x, y, ww, bb in ((q, out[0], w[0], w[1]), (k, out[1], w[2], w[3])):
        f = None if inv is None else host(inv)
        ref = orc.norm_rope(host(x), norm, None if ww is None else host(ww), None if bb is None else host(bb), 1e-5, None if several else rope, r, f, pos)
        if several:
            ref = orc8.rotate_axes(ref, rope, f, pos, axes)
        amax = np.abs(ref).max(-1, keepdims=True) * np.sqrt(2)
        assert np.all(np.abs(host(y) - ref) <= HALF[dt] * np.abs(ref) + 2e-5 * amax + 2.0 ** -25)
    major = binding.qk_norm_rope(q, k, v, head_major=True, **kw)
    assert all(a.is_contiguous() and torch.equal(a.transpose(0, 1), b) for a, b in zip(major, out))


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d,hq,hkv,n", [(64, 3, 3, COUNTS[0]), (128, 9, 1, COUNTS[0]), (64, 16, 2, COUNTS[1]), (128, 4, 2, COUNTS[2]), (64, 5, 1, COUNTS[3]), (128, 32, 8, 3701)])
@pytest.mark.parametrize("norm,rope,rotary", [("rms", "half", None), ("layer", "2d", None), (None, "pairs", None), ("rms", "half", 32),
                                              ("layer", "pairs", 24), ("layer", None, None), ("rms", None, None), (None, "2d", None), (None, None, None)])
def test_norm_rope(dtype, d, hq, hkv, n, norm, rope, rotary):
    check(dtype, d, hq, hkv, n, norm, rope, rotary, None)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d,hq,hkv,n", [(64, 3, 3, COUNTS[0]), (128, 5, 1, COUNTS[1]), (64, 8, 2, COUNTS[2]), (128, 4, 1, COUNTS[3])])
@pytest.mark.parametrize("norm,rope,rotary,several", [("rms", "half", None, 3), ("layer", "pairs", None, 2), (None, "pairs", 24, 3), ("rms", "half", 32, 8),
                                                      (None, "half", None, 1)])
def test_axes(dtype, d, hq, hkv, n, norm, rope, rotary, several):
    check(dtype, d, hq, hkv, n, norm, rope, rotary, several)
