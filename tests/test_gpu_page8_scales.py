"""The operators over a shared pool of 8-bit pages where one page differs from its neighbours (values beside an outlier, scales far apart).
Tolerances are those of test_gpu_page8_ops.py."""
import numpy as np
import pytest
import torch

from oracle import page_oracle as orc4
from paper_2602_21780_b200 import binding
from tests.test_gpu_page8_ops import ATTN, DT, PAGE, WIDE, Server, host, ints

pytestmark = pytest.mark.gpu


def fill(sv, x, v, new):
    """One sequence, the same x and v for every key/value head: all but the last `new` tokens in one call, then those; x is what channel 0
    of the keys gives a logit of the queries that ask() makes."""
    k = 0.1 * sv.rnd(len(x), sv.hkv, sv.d)
    k[..., 0] = torch.as_tensor(x, dtype=torch.float32, device="cuda")[:, None]
    k, v, at = k.to(sv.dt), v[:, None].expand(-1, sv.hkv, -1).to(sv.dt), 0
    for n in (len(x) - new, new):
        plan = binding.page_plan(sv.len, ints([n]), sv.table, sv.ring, sv.state, n)
        sv.len, sv.state = plan.total_len, plan.ring_state
        rows = (k[at:at + n], v[at:at + n].contiguous())
        binding.page8_append(sv.pages, *rows, plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
        sv.note([n], plan, *rows)
        at += n
    return plan


def ask(sv, plan, new, group, channels=slice(None)):
    """Attention of queries whose first channel is 8, against the oracle, over some of the channels."""
    q = sv.rnd(new, group * sv.hkv, sv.d)
    q[..., 0] = 8
    q = q.to(sv.dt)
    out = host(binding.page8_attention(q, sv.pages, sv.table, plan.cu_new, plan.total_len, new, scale=0.125))[..., channels]
    held = [(r.k, r.v) for r in sv.ref[0]]
    ref = np.stack([orc4.attention(host(q[:, h]), *held[h // group], 0.125) for h in range(q.shape[1])], 1)[..., channels]
    err, size = np.linalg.norm(out - ref, axis=-1), np.linalg.norm(ref, axis=-1)
    assert np.all(np.isfinite(out))
    assert np.linalg.norm(err) <= ATTN[sv.dt] * np.linalg.norm(size), np.linalg.norm(err) / np.linalg.norm(size)
    assert np.all(err <= 3 * ATTN[sv.dt] * size)


# few query rows a head; more, by either kernel
KERNELS = [(1, 80), (40, 80), (40, WIDE)]


@pytest.mark.parametrize("new,width", KERNELS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("big,page", [(512.0, 20), (4096.0, 20), (60000.0, 20), (60000.0, 0)])
def test_a_page_whose_largest_value_nobody_attends_to(new, width, d, dtype, big, page):
    # A page holds a token with nearly all of the attention and values near zero, and one with a value of `big` and no attention:
    # the result is what 4096 other tokens give it, each with e^-11 of the weight.  Their weights stand at 2^-16 of the largest one, which leaves
    # fp16 its full significand in both kernels, so that the usual tolerance holds; the heavy token's own weight, if it is rounded
    # for the sum, costs 2^-11 of the result, which the weights' share of the tolerance covers.
    sv = Server(1, 1, d, dtype, pages=70, width=width, seed=d + page)
    n = 4096 + new
    x, v = 0.3 * np.random.default_rng(page).standard_normal(n), sv.rnd(n, d) + 1
    x[page * PAGE + 3], x[page * PAGE + 7] = 11, -60
    v[page * PAGE + 3] = 1e-3 * sv.rnd(d)
    v[page * PAGE + 7, 5] = big
    plan = fill(sv, x, v, new)
    ask(sv, plan, new, 4)
    ask(sv, plan, new, 4, np.arange(d) != 5)


@pytest.mark.parametrize("new,width", KERNELS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,small", [("fp16", 2.0 ** -10), ("bf16", 2.0 ** -10), ("bf16", 2.0 ** -60), ("bf16", 2.0 ** -68)])
def test_small_values_between_large_ones_that_nobody_attends_to(new, width, d, dtype, small):
    # every other page has values of 60000 and no attention (e^-60), those between have what is attended to: scales 2^25 and more apart
    sv = Server(1, 1, d, dtype, pages=70, width=width, seed=3 * d)
    n = 30 * PAGE + new
    odd = np.arange(n) // PAGE % 2 == 1
    x = np.where(odd, -60 if small > 1e-6 else -150, 0.5 * np.random.default_rng(d).standard_normal(n))
    v = (sv.rnd(n, d) + 1).clamp(-3, 3) * torch.as_tensor(np.where(odd, 20000.0, small), dtype=torch.float32, device="cuda")[:, None]
    ask(sv, fill(sv, x, v, new), new, 4)


@pytest.mark.parametrize("new,width", KERNELS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,size", [("fp16", 1.0), ("bf16", 1.0), ("bf16", 2.0 ** -68)])
def test_pages_of_zeros_between_others(new, width, d, dtype, size):
    # pages with the smallest scale that there is, attended to like the others
    sv = Server(1, 1, d, dtype, pages=70, width=width, seed=5 * d)
    n = 40 * PAGE + new
    there = np.arange(n) // PAGE % 3 != 1
    v = (sv.rnd(n, d) + 1) * torch.as_tensor(there * size, dtype=torch.float32, device="cuda")[:, None]
    ask(sv, fill(sv, 0.5 * np.random.default_rng(d).standard_normal(n), v, new), new, 4)


@pytest.mark.parametrize("new,width", KERNELS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("sizes", [(6, -10, 8, -3), (-10, 6, -10, 7), (8, -7, -10, 8)])
def test_runs_of_pages_of_different_scales(new, width, d, dtype, sizes):
    # 37 pages of each size, and weights that give each size its share of the result: 2^18 apart, fp16's full significand in both kernels
    sv = Server(1, 1, d, dtype, pages=160, width=max(width, 160), seed=d - sizes[0])
    n = 37 * PAGE * len(sizes) + new
    size = np.repeat(sizes, 37 * PAGE).tolist() + [sizes[-1]] * new
    x = 0.3 * np.random.default_rng(d).standard_normal(n) - np.log(2.0) * np.array(size)
    v = (sv.rnd(n, d) + 1) * torch.tensor(size, device="cuda", dtype=torch.float32).exp2()[:, None]
    ask(sv, fill(sv, x, v, new), new, 4)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("order", [1, -1])
def test_scales_that_change_within_a_span(d, dtype, order):
    # Enough work that a block walks through 50 and more pages of a unit: runs of one size, and between two of them pages that alternate with
    # ones whose large values nobody attends to (60).
    sizes = ([6] * 40 + [60, -10] * 15 + [-10] * 40 + [8] * 40)[::order]
    new = 400
    sv = Server(1, 8, d, dtype, pages=170, width=170, seed=d + order)
    size = np.array(np.repeat(sizes, PAGE).tolist() + [sizes[-1]] * new)
    n = len(size)
    x = np.where(size == 60, -60, 0.3 * np.random.default_rng(d).standard_normal(n) - np.log(2.0) * size)
    v = (sv.rnd(n, d) + 1).clamp(-3, 3) * torch.as_tensor(np.where(size == 60, 20000.0, 2.0 ** np.minimum(size, 20)), dtype=torch.float32, device="cuda")[:, None]
    ask(sv, fill(sv, x, v, new), new, 4)
