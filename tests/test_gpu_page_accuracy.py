"""How exact the attention over 4-bit pages is, at tolerances that its roundings alone explain.

Tolerances.  The roundings of both kernels were emulated in float64 with sums that are exact, on inputs of the distributions
below (48 query rows, three seeds), as the relative 2-norm of the error over all rows:
  few rows   P, P s, q s and, at fp16, z + 8 s to float16; at fp16 codes around their middle
  many rows  keys and values to float16, P to float16 in the numerator alone
  both       the result to its type
and came to, for 704 tokens of zero mean, the larger of head_dim 64 and 128,
                          few fp16   few bf16   many fp16  many bf16
  queries of size 0.1     4.04e-4    1.85e-3    3.84e-4    1.73e-3       (values' roundings)
  queries of size 1       5.53e-4    2.03e-3    5.27e-4    1.77e-3       (and the logits')
without the centring of the codes few fp16 would be 7.11e-4 and 9.04e-4; for 20 480 tokens of mean 3 and queries of size 1
                          1.89e-4    1.52e-3    1.89e-4    1.52e-3       (the result's rounding: about half a step / sqrt(3))
A fifth is added for other inputs and for the roundings of float32 sums: 704 tokens have 11 pages and 44 products in a sum,
each within 2^-20 of its largest partial sum.
"""
import numpy as np
import pytest
import torch

from oracle import page_oracle as orc
from paper_2602_21780_b200 import binding
from tests.test_gpu_page_ops import Server, host, ints

pytestmark = pytest.mark.gpu

FEW, MANY = (12, 4), (12, 10)               # query heads over one key/value head, new tokens: 48 rows a head, 120 rows


def error(dtype, d, shape, tokens, size, mean):
    hq, new = shape
    sv = Server(1, 1, d, dtype, pages=tokens // 64 + 3, width=tokens // 64 + 3, seed=d + new)
    for n in (tokens, new):
        plan = binding.page_plan(sv.len, ints([n]), sv.table, sv.ring, sv.state, n)
        sv.len, sv.state = plan.total_len, plan.ring_state
        k = ((sv.rnd(n, 1, d) + sv.mu) * sv.w).to(sv.dt)
        v = (sv.rnd(n, 1, d) + mean).to(sv.dt)
        binding.page_append(sv.pages, sv.tail, k, v, plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
        sv.ref[0][0].append(host(k[:, 0]), host(v[:, 0]))
    q = (sv.rnd(new, hq, d) * size).to(sv.dt)
    out = host(binding.page_attention(q, sv.pages, sv.tail, sv.table, plan.cu_new, plan.total_len, new))
    r = sv.ref[0][0]
    ref = np.stack([orc.attention(host(q[:, h]), r.k, r.v, d ** -0.5) for h in range(hq)], 1)
    return np.linalg.norm(out - ref) / np.linalg.norm(ref)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape,dtype,size,emulated", [(FEW, "fp16", 0.1, 4.04e-4), (FEW, "fp16", 1.0, 5.53e-4), (FEW, "bf16", 0.1, 1.85e-3),
                                                       (FEW, "bf16", 1.0, 2.03e-3), (MANY, "fp16", 0.1, 3.84e-4), (MANY, "fp16", 1.0, 5.27e-4),
                                                       (MANY, "bf16", 0.1, 1.73e-3), (MANY, "bf16", 1.0, 1.77e-3)])
def test_values_of_zero_mean(d, shape, dtype, size, emulated):
    assert error(dtype, d, shape, 704, size, 0.0) <= 1.2 * emulated


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", [FEW, MANY])
@pytest.mark.parametrize("dtype,emulated", [("fp16", 1.89e-4), ("bf16", 1.52e-3)])
def test_a_long_sequence_of_values_with_a_mean(d, shape, dtype, emulated):
    assert error(dtype, d, shape, 20480, 1.0, 3.0) <= 1.2 * emulated
