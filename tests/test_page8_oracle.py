"""Pins of the oracle of the 8-bit pages and the host-side refusals of their entry points (no GPU needed)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import page8_oracle as orc
from paper_2602_21780_b200 import binding

A = 1 << 20            # an aligned address that is never read: every call below is refused before a launch


def test_e4m3_against_torch():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(orc.VALUES, want, equal_nan=True)
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.standard_normal(20000) * 10.0 ** rng.uniform(-4, 2.5, 20000), (orc.VALUES[1:127] + orc.VALUES[:126]) / 2,
                        orc.VALUES[:127], [0.0, -0.0, 448, 500, -1e9, 2.0 ** -10, 3 * 2.0 ** -10]])
    x = x.astype(np.float32)
    want = torch.from_numpy(np.clip(x, -448, 448)).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(orc.nearest(x), want)


def test_scale_by_hand():
    assert [orc.exponent(a) for a in (448, 448.1, 224, 1.75, 65504, 1e9, 0, 1e-30)] == [0, 1, -1, -8, 8, 8, -80, -80]
    b = orc.Block(2)
    b.append([[448, 2.0 ** -6]])
    b.append([[4480, 0.3]])                 # needs 2^4: 448 -> 28, 2^-6 -> 2^-10, which is half the smallest code: to even, 0
    assert b.e == 4 and np.array_equal(b.codes, [[28, 0], [280 + 8, 0.01953125]])
    b.append([[1, 1]])
    assert b.e == 4 and np.array_equal(b.values()[2], [1, 1])


def test_every_code_has_a_place_of_its_own():
    for d in (64, 128):
        tok, ch = np.arange(64)[:, None], np.arange(d)[None, :]
        k, v = (np.broadcast_to(f(tok, ch, d), (64, d)).ravel() for f in (orc.key_place, orc.value_place))
        assert sorted(k) == list(range(64 * d)) and sorted(v) == list(range(64 * d + 32, 128 * d + 32))


def test_selection_by_hand():
    ones = np.ones(4)
    means = [(ones.astype(int) * m, 1.0) for m in (1, 9, 3, 9, 5, 2, 7, 1)]
    assert orc.select(ones[None], means, 7, 5, 1, 2).__len__() == 5
    assert orc.select(ones[None], means, 7, 5, 1, 2) == [0, 1, 3, 6, 7]           # 9, 9 of pages 1 to 5
    assert orc.select(ones[None], means, 7, 4, 1, 2) == [0, 1, 6, 7]              # equal scores: the lower page
    assert orc.select(-ones[None], means, 7, 4, 0, 1) == [0, 2, 5, 7]             # the others' order, among pages 0 to 6: 1, 2, 3
    assert orc.select(ones[None], means, 2, 5, 1, 2) == [0, 1, 2, -1, -1]
    assert orc.select(ones[None], [None] + means[1:], 7, 3, 0, 1) == [1, 3, 7]
    two = np.stack([ones, -3 * ones])       # a head each way: the larger of both
    assert orc.select(two, means, 7, 3, 0, 1) == [1, 3, 7]


def test_mean_key_is_near_the_mean():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((64, 128)) + rng.standard_normal(128)
    b = orc.Block(128)
    b.append(x)
    codes, factor = orc.mean_key(b.codes, b.e)
    assert np.abs(codes).max() == 127
    assert np.all(np.abs(codes * factor / 127 - b.values().mean(0)) <= factor / 127 / 2 * 1.0001)


# ------------------------------------------------------------------ refusals
def _pool(**kw):
    v = dict(records=A, n_pages=10, kv_heads=2, head_dim=64, dtype=0)
    v.update(kw)
    return binding._Page8Pool(**v)


APPEND = dict(K=A, V=A, ks=128, vs=128, n=3, slot=A, seq=A, cu=A, total=A, seqs=2)
READ = dict(table=A, width=5, total=A, seqs=2, seq=A, pos=A, n=3, K=A, V=A)
ATTN = dict(Q=A, qs=256, n=3, heads=4, table=A, width=5, cu=A, total=A, slot=None, seqs=2, max_new=3, scale=0.1, window=0, out=A, ws=A, wb=1 << 40)
SELECT = dict(Q=A, qs=256, n=3, heads=4, table=A, width=5, seqs=2, seq=A, pos=A, slot=None, top=4, first=1, recent=2, out=A)
SELECTED = dict(Q=A, qs=256, n=3, heads=4, table=A, width=5, seqs=2, seq=A, pos=A, sel=A, top=4, scale=0.1, out=A, ws=A, wb=1 << 40)


def call(name, args, pool=None):
    return getattr(binding.load(), name)(C.byref(pool or _pool()), *args.values(), None)


@pytest.mark.parametrize("bad,code", [(dict(records=None), 1), (dict(n_pages=0), 1), (dict(kv_heads=0), 1), (dict(kv_heads=65536), 1), (dict(head_dim=96), 1),
                                      (dict(dtype=2), 1), (dict(records=A + 8), 2), (dict(n_pages=(1 << 25) + 1), 9)])
def test_bad_pools_are_refused(bad, code):
    for name, args in (("append", APPEND), ("read", READ), ("attention", ATTN), ("select", SELECT), ("attention_selected", SELECTED)):
        assert call("xsv_page8_" + name, args, _pool(**bad)) == code


@pytest.mark.parametrize("bad,code", [(dict(K=None), 1), (dict(V=None), 1), (dict(n=-1), 1), (dict(seqs=0), 1), (dict(seqs=8193), 1),
                                      (dict(slot=None), 1), (dict(seq=None), 1), (dict(cu=None), 1), (dict(total=None), 1),
                                      (dict(ks=120), 1), (dict(vs=64), 1), (dict(ks=132), 2), (dict(K=A + 8), 2), (dict(n=0), 0)])
def test_append_arguments(bad, code):
    assert call("xsv_page8_append", {**APPEND, **bad}) == code


@pytest.mark.parametrize("bad,code", [(dict(table=None), 1), (dict(width=0), 1), (dict(total=None), 1), (dict(seqs=8193), 1), (dict(seq=None), 1),
                                      (dict(pos=None), 1), (dict(n=-2), 1), (dict(K=None), 1), (dict(V=A + 4), 2), (dict(n=0), 0)])
def test_read_arguments(bad, code):
    assert call("xsv_page8_read", {**READ, **bad}) == code


@pytest.mark.parametrize("bad,code", [(dict(Q=None), 1), (dict(heads=3), 1), (dict(heads=1), 1), (dict(n=-1), 1), (dict(table=None), 1),
                                      (dict(width=0), 1), (dict(cu=None), 1), (dict(total=None), 1), (dict(seqs=0), 1), (dict(max_new=-1), 1),
                                      (dict(scale=0.0), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(window=-1), 1),
                                      (dict(out=None), 1), (dict(ws=None), 1), (dict(wb=16), 1), (dict(qs=128), 1), (dict(qs=260), 2),
                                      (dict(Q=A + 2), 2), (dict(out=A + 8), 2), (dict(ws=A + 4), 2), (dict(width=1 << 25), 9),
                                      (dict(n=0), 0), (dict(max_new=0), 0)])
def test_attention_arguments(bad, code):
    assert call("xsv_page8_attention", {**ATTN, **bad}) == code


@pytest.mark.parametrize("bad,code", [(dict(Q=None), 1), (dict(heads=3), 1), (dict(heads=1), 1), (dict(n=-1), 1), (dict(table=None), 1), (dict(width=0), 1),
                                      (dict(seqs=0), 1), (dict(seqs=8193), 1), (dict(seq=None), 1), (dict(pos=None), 1), (dict(out=None), 1),
                                      (dict(top=0), 1), (dict(first=-1), 1), (dict(recent=0), 1), (dict(first=3), 1), (dict(first=1 << 30), 1), (dict(recent=5), 1),
                                      (dict(qs=128), 1), (dict(qs=260), 2), (dict(Q=A + 2), 2), (dict(top=1025), 9), (dict(width=32769), 9),
                                      (dict(heads=2 * 129, qs=2 * 129 * 64), 9), (dict(n=0), 0)])
def test_select_arguments(bad, code):
    assert call("xsv_page8_select", {**SELECT, **bad}) == code


@pytest.mark.parametrize("bad,code", [(dict(Q=None), 1), (dict(heads=3), 1), (dict(n=-1), 1), (dict(table=None), 1), (dict(width=0), 1), (dict(seqs=0), 1),
                                      (dict(seq=None), 1), (dict(pos=None), 1), (dict(sel=None), 1), (dict(top=0), 1), (dict(scale=0.0), 1),
                                      (dict(scale=float("nan")), 1), (dict(out=None), 1), (dict(ws=None), 1), (dict(wb=16), 1), (dict(qs=128), 1),
                                      (dict(qs=260), 2), (dict(Q=A + 2), 2), (dict(out=A + 8), 2), (dict(ws=A + 4), 2), (dict(width=1 << 25), 9),
                                      (dict(top=1025), 9), (dict(n=0), 0)])
def test_selected_arguments(bad, code):
    assert call("xsv_page8_attention_selected", {**SELECTED, **bad}) == code


def test_workspace_queries():
    f, g = binding.load().xsv_page8_attention_workspace, binding.load().xsv_page8_attention_selected_workspace
    assert f(1, 1, 1, 16, 16, 64) > 0 and f(64, 64, 1, 32, 8, 128) > 0 and f(4000, 3, 2000, 32, 8, 128) > f(64, 64, 1, 32, 8, 128)
    for bad in ((0, 1, 1, 4, 2, 64), (1, 0, 1, 4, 2, 64), (1, 8193, 1, 4, 2, 64), (1, 1, 0, 4, 2, 64), (1, 1, 1, 3, 2, 64), (1, 1, 1, 4, 0, 64),
                (1, 1, 1, 4, 2, 96)):
        assert f(*bad) == 0
    assert g(16, 16, 64) > 0 and g(32, 2, 128) > g(16, 2, 128) > 0 and g(3, 2, 64) == g(4, 0, 64) == g(4, 2, 96) == 0


AXES = dict(q=A, k=A, v=A, qs=256, ks=128, vs=128, n=3, hq=4, hkv=2, d=64, dtype=1, norm=1, qw=A, qb=None, kw=A, kb=None, eps=1e-6,
            rope=1, rot=64, freq=A, pos=A, axes=A, n_axes=3, layout=0, qo=A, ko=A, vo=A)


@pytest.mark.parametrize("bad,code", [(dict(rope=0), 1), (dict(rope=3), 1), (dict(n_axes=0), 1), (dict(n_axes=9), 1), (dict(axes=None), 1), (dict(axes=A + 2), 2),
                                      (dict(pos=None), 1), (dict(freq=None), 1), (dict(rot=60), 1), (dict(q=None), 1), (dict(pos=A + 2), 2), (dict(ks=132), 2),
                                      (dict(n=0, axes=None), 0)])
def test_axes_arguments(bad, code):
    assert binding.load().xsv_qk_norm_rope_axes(*{**AXES, **bad}.values(), None) == code


def test_binding_refuses_tensors_it_cannot_take():
    x, i = torch.zeros(3, 2, 64, dtype=torch.float16), torch.zeros(3, dtype=torch.int32)
    pages = torch.zeros(4, 2, 130 * 64, dtype=torch.uint8)
    for call_ in (lambda: binding.page8_append(pages, x, x, i, i, i, i), lambda: binding.page8_read(pages, i[None], i, i, i, torch.float16),
                  lambda: binding.page8_attention(x, pages, i[None], i, i, 1), lambda: binding.page8_select(x, pages, i[None], i, i, 4),
                  lambda: binding.page8_attention_selected(x, pages, i[None], i, i, i.view(1, 1, 3))):
        with pytest.raises(ValueError, match="CUDA"):
            call_()


def test_select_without_pages_that_are_not_there():
    means = [(np.array([p, 0]), 1.0) for p in range(12)]                     # the later, the better
    q, lost = np.array([[127.0, 0.0]]), [p not in (0, 8, 11) for p in range(12)]
    gone = [m if there else None for m, there in zip(means, lost)]
    assert orc.select(q, means, 11, 6, 2, 3) == [0, 1, 8, 9, 10, 11]
    assert orc.select(q, gone, 11, 6, 2, 3, lost) == [1, 5, 6, 7, 9, 10]
    assert orc.select(q, [None] * 12, 11, 3, 1, 2, [False] * 12) == [-1] * 3
    assert orc.select(q, gone, 1, 6, 2, 3, lost) == [1] + [-1] * 5
