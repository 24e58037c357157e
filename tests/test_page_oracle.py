"""Pins of the page oracle and the host-side refusals of the page entry points (no GPU needed)."""
import ctypes as C

import numpy as np
import pytest

from oracle import page_oracle as orc
from paper_2602_21780_b200 import binding

A = 1 << 20            # an aligned address that is never read: every call below is refused before a launch


def test_every_code_has_a_place_of_its_own():
    for d in (64, 128):
        tok, ch = np.arange(64)[:, None], np.arange(d)[None, :]
        for (byte, shift), lo in ((orc.key_place(tok, ch), 0), (orc.value_place(tok, ch, d), 32 * d)):
            at = np.broadcast_to(byte * 2 + shift // 4, (64, d))
            assert sorted(at.ravel()) == list(range(2 * lo, 2 * lo + 64 * d))


def test_quantiser_rounds_parameters_outwards():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((50, 64)) * 10.0 ** rng.uniform(-6, 4, (50, 1)) + rng.standard_normal((50, 1)) * 100
    x[0] = 3.25                                     # a constant group
    x[1] = np.linspace(-65504, 65504, 64)
    x[2, :] = 0
    c, s, z = orc.quantise(x, 1)
    assert np.all(z <= x.min(1, keepdims=True)) and np.all(s > 0) and c.min() >= 0 and c.max() <= 15
    assert np.all(np.abs(c * s + z - np.clip(x, -65504, 65504)) <= s / 2 * (1 + 1e-12))
    assert np.array_equal(s.astype(np.float16).astype(np.float64), s) and np.array_equal(z.astype(np.float16).astype(np.float64), z)
    assert np.all(c[0] * s[0] + z[0] == 3.25) and s[2, 0] == 1


def test_plan_by_hand():
    # 70 + 60 tokens: one page held twice (pages 4, 5), 130 needs a third (page 9); sequence 1 ends and gives 7 back;
    # sequence 2 starts with 1 token (page 3)
    table = np.array([[4, 5, -1], [7, -1, -1], [-1, -1, -1]], np.int32)
    ring = np.array([3, 0, 0, 0, 0, 0, 0, 0, 0, 9], np.int32)
    state, cu, total, slot, seq, pos = orc.plan([70, 10, 0], [60, -1, 1], table, ring, [9, 2], 64)
    assert table.tolist() == [[4, 5, 9], [7, -1, -1], [3, -1, -1]] and state.tolist() == [1, 1, 0, 61]
    assert ring[1] == 7 and cu.tolist() == [0, 60, 60, 61] and total.tolist() == [130, 0, 1]
    assert slot[:2].tolist() == [5 * 64 + 6, 5 * 64 + 7] and slot[57:64].tolist() == [5 * 64 + 63, 9 * 64, 9 * 64 + 1, 3 * 64, -1, -1, -1]
    assert seq[60:].tolist() == [2, -1, -1, -1] and pos[60:].tolist() == [0, 0, 0, 0]


# ------------------------------------------------------------------ refusals
def _pool(**kw):
    v = dict(records=A, k_tail=A, n_pages=10, max_seqs=4, kv_heads=2, head_dim=64, dtype=0)
    v.update(kw)
    return binding._PagePool(**v)


BAD_POOLS = [(dict(records=None), 1), (dict(k_tail=None), 1), (dict(n_pages=0), 1), (dict(max_seqs=0), 1), (dict(kv_heads=0), 1),
             (dict(head_dim=96), 1), (dict(dtype=2), 1), (dict(records=A + 8), 2), (dict(k_tail=A + 2), 2),
             (dict(n_pages=(1 << 25) + 1), 9), (dict(max_seqs=8193), 9)]


@pytest.mark.parametrize("bad,code", BAD_POOLS)
def test_bad_pools_are_refused(bad, code):
    lib, p = binding.load(), _pool(**bad)
    assert lib.xsv_page_append(C.byref(p), A, A, 128, 128, 3, A, A, A, A, 2, None) == code
    assert lib.xsv_page_read(C.byref(p), A, 5, A, 2, A, A, 3, A, A, None) == code
    assert lib.xsv_page_attention(C.byref(p), A, 256, 3, 4, A, 5, A, A, 2, 3, 1.0, 0, A, A, 1 << 40, None) == code


APPEND = dict(K=A, V=A, ks=128, vs=128, n=3, slot=A, seq=A, cu=A, total=A, seqs=2)


@pytest.mark.parametrize("bad,code", [(dict(K=None), 1), (dict(V=None), 1), (dict(n=-1), 1), (dict(seqs=0), 1), (dict(seqs=5), 1),
                                      (dict(slot=None), 1), (dict(seq=None), 1), (dict(cu=None), 1), (dict(total=None), 1),
                                      (dict(ks=120), 1), (dict(vs=64), 1), (dict(ks=132), 2), (dict(K=A + 8), 2), (dict(n=0), 0)])
def test_append_arguments(bad, code):
    a, p = {**APPEND, **bad}, _pool()
    assert binding.load().xsv_page_append(C.byref(p), *a.values(), None) == code


READ = dict(table=A, width=5, total=A, seqs=2, seq=A, pos=A, n=3, K=A, V=A)


@pytest.mark.parametrize("bad,code", [(dict(table=None), 1), (dict(width=0), 1), (dict(total=None), 1), (dict(seqs=9), 1), (dict(seq=None), 1),
                                      (dict(pos=None), 1), (dict(n=-2), 1), (dict(K=None), 1), (dict(V=A + 4), 2), (dict(n=0), 0)])
def test_read_arguments(bad, code):
    a, p = {**READ, **bad}, _pool()
    assert binding.load().xsv_page_read(C.byref(p), *a.values(), None) == code


ATTN = dict(Q=A, qs=256, n=3, heads=4, table=A, width=5, cu=A, total=A, seqs=2, max_new=3, scale=0.1, window=0, out=A, ws=A, wb=1 << 40)


@pytest.mark.parametrize("bad,code", [(dict(Q=None), 1), (dict(heads=3), 1), (dict(heads=1), 1), (dict(n=-1), 1), (dict(table=None), 1),
                                      (dict(width=0), 1), (dict(cu=None), 1), (dict(total=None), 1), (dict(seqs=0), 1), (dict(max_new=-1), 1),
                                      (dict(scale=0.0), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(window=-1), 1),
                                      (dict(out=None), 1), (dict(ws=None), 1), (dict(wb=16), 1), (dict(qs=128), 1), (dict(qs=260), 2),
                                      (dict(Q=A + 2), 2), (dict(out=A + 8), 2), (dict(ws=A + 4), 2), (dict(width=1 << 25), 9),
                                      (dict(n=0), 0), (dict(max_new=0), 0)])
def test_attention_arguments(bad, code):
    a, p = {**ATTN, **bad}, _pool()
    assert binding.load().xsv_page_attention(C.byref(p), *a.values(), None) == code


def test_attention_workspace_query():
    f = binding.load().xsv_page_attention_workspace
    assert f(1, 1, 1, 16, 16, 64) > 0 and f(64, 64, 1, 32, 8, 128) > 0
    assert f(4000, 3, 2000, 32, 8, 128) > f(64, 64, 1, 32, 8, 128)
    for bad in ((0, 1, 1, 4, 2, 64), (1, 0, 1, 4, 2, 64), (1, 8193, 1, 4, 2, 64), (1, 1, 0, 4, 2, 64), (1, 1, 1, 3, 2, 64), (1, 1, 1, 4, 0, 64),
                (1, 1, 1, 4, 2, 96)):
        assert f(*bad) == 0


PLAN = dict(cached=A, new=A + 64, n=2, table=A, width=3, ring=A, pages=9, state=A, state_out=A + 64, cu=A + 128, total=A + 256,
            slot=A, seq=A, pos=A, most=5)


@pytest.mark.parametrize("bad,code", [(dict(cached=None), 1), (dict(new=None), 1), (dict(n=0), 1), (dict(table=None), 1), (dict(width=0), 1),
                                      (dict(ring=None), 1), (dict(pages=0), 1), (dict(state=None), 1), (dict(state_out=None), 1),
                                      (dict(state_out=A), 1), (dict(cu=None), 1), (dict(total=None), 1), (dict(total=A), 1),
                                      (dict(total=A + 64), 1), (dict(slot=None), 1), (dict(seq=None), 1), (dict(pos=None), 1),
                                      (dict(most=-1), 1), (dict(n=8193), 9), (dict(pages=(1 << 25) + 1), 9)])
def test_plan_arguments(bad, code):
    assert binding.load().xsv_page_plan(*{**PLAN, **bad}.values(), None) == code


NORM = dict(q=A, k=A, v=A, qs=256, ks=128, vs=128, n=3, hq=4, hkv=2, d=64, dtype=1, norm=1, qw=A, qb=None, kw=A, kb=None, eps=1e-6,
            rope=1, rot=64, freq=A, pos=A, layout=0, qo=A, ko=A, vo=A)


@pytest.mark.parametrize("bad,code", [(dict(q=None), 1), (dict(qo=None), 1), (dict(vo=None), 1), (dict(n=-1), 1), (dict(hq=0), 1), (dict(hkv=0), 1),
                                      (dict(hq=-1), 1), (dict(d=80), 1), (dict(dtype=2), 1), (dict(norm=3), 1), (dict(norm=-1), 1), (dict(rope=4), 1),
                                      (dict(layout=2), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(rot=60), 1), (dict(rot=72), 1),
                                      (dict(rot=0), 1), (dict(rope=3, rot=32), 1), (dict(freq=None), 1), (dict(pos=None), 1), (dict(freq=A + 2), 2),
                                      (dict(qs=248), 1), (dict(qs=260), 2), (dict(q=A + 8), 2), (dict(qw=A + 4), 2), (dict(ko=A + 2), 2),
                                      (dict(n=0), 0), (dict(q=None, k=None, v=None, qo=None, ko=None, vo=None), 1)])
def test_norm_rope_arguments(bad, code):
    assert binding.load().xsv_qk_norm_rope(*{**NORM, **bad}.values(), None) == code


def test_binding_refuses_tensors_it_cannot_take():
    import torch
    x = torch.zeros(3, 2, 64, dtype=torch.float16)
    with pytest.raises(ValueError, match="CUDA"):
        binding.qk_norm_rope(x, x)
    with pytest.raises(ValueError, match="unknown"):
        binding.qk_norm_rope(x, x, norm="batch")
    with pytest.raises(ValueError, match="CUDA"):
        binding.page_plan(*[torch.zeros(3, dtype=torch.int32)] * 5, 3)
