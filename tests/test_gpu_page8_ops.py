"""The operators over a shared pool of 8-bit pages, and the rotation by several positions, against the float64 oracle, on the GPU.

Tolerances.  A result that is rounded once to the output type is off by at most half a step, 2^-11 relative for fp16 and 2^-8
for bf16.
  rotation: besides that, float32 arithmetic on a row whose largest element is A: below 2e-5 * A (128 * 2^-24 on a mean of
    squares, half of it on the root, 8 * 2^-24 for rotation, angle and products).
  append, read: codes, scales and mean keys are those of the oracle, bit for bit; a value read back is a code times a power of
    two, exact in both types but for fp16's range (2^-25 below it, 65504 above it).
  select: page numbers are those of the oracle.
  attention: queries and codes are exact as fp16 operands; every weight P is rounded to fp16, at most 2^-11 of itself,
    independently, where the output is the sum of the same terms: 2^-11 of its 2-norm.  With the output's own half step that is
    2^-10 of the 2-norm over all rows for fp16 and 2^-8 + 2^-11 for bf16.  A single row's terms may cancel: three times that.
"""
import numpy as np
import pytest
import torch

from oracle import page8_oracle as orc
from oracle import page_oracle as orc4
from paper_2602_21780_b200 import binding

pytestmark = pytest.mark.gpu

PAGE = 64
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
ATTN = {torch.float16: 2.0 ** -10, torch.bfloat16: 2.0 ** -8 + 2.0 ** -11}
DT = {"fp16": torch.float16, "bf16": torch.bfloat16}


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def host(t):
    return t.double().cpu().numpy()


def near(got, ref, dt):
    err, size = np.linalg.norm(got - ref, axis=-1), np.linalg.norm(ref, axis=-1)
    assert np.all(np.isfinite(got))
    assert np.linalg.norm(err) <= ATTN[dt] * np.linalg.norm(size) + 1e-30
    assert np.all(err <= 3 * ATTN[dt] * size + 1e-6 * np.abs(ref).max(initial=0.0))


# ------------------------------------------------------------------------------------------------ rotation by several positions
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d,hq,hkv,n", [(64, 3, 3, 1), (128, 8, 1, 1), (64, 16, 16, 261), (128, 20, 4, 700)])
@pytest.mark.parametrize("norm,rope,rotary,several", [("rms", "half", None, 3), ("layer", "pairs", None, 2), (None, "pairs", 24, 3), ("rms", "half", 32, 8),
                                                      (None, "half", None, 1)])
def test_axes(dtype, d, hq, hkv, n, norm, rope, rotary, several):
    dt, r = DT[dtype], rotary or d
    g = torch.Generator(device="cuda").manual_seed(d + n)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    fused = (rnd(n, (hq + 2 * hkv) * d + 8) * (0.1 + 3 * torch.rand(n, 1, device="cuda", generator=g)) + 0.3).to(dt)
    q, k, v = (fused[:, a * d:b * d].view(n, b - a, d) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
    w = [(1 + 0.3 * rnd(d)).to(dt), None, (1 + 0.3 * rnd(d)).to(dt), (0.2 * rnd(d)).to(dt)] if norm else [None] * 4
    rng = np.random.default_rng(n)
    inv, pos = 10000.0 ** (-torch.arange(r // 2, device="cuda") / (r / 2)), rng.integers(-5, 2_000_000, (n, several))
    axes = rng.integers(0, several, r // 2)
    if several == 3:
        axes[rng.integers(0, r // 2, 2)] = (-1, 3)               # no such position: not rotated
    out = binding.qk_norm_rope(q, k, v, norm=norm, q_weight=w[0], q_bias=w[1], k_weight=w[2], k_bias=w[3], eps=1e-5, rope=rope, inv_freq=inv,
                               positions=ints(pos), axes=ints(axes))
    assert torch.equal(out[2], v)
    for x, y, ww, bb in ((q, out[0], w[0], w[1]), (k, out[1], w[2], w[3])):
        ref = orc4.norm_rope(host(x), norm, None if ww is None else host(ww), None if bb is None else host(bb), 1e-5, None, r, None, None)
        ref = orc.rotate_axes(ref, rope, host(inv), pos, axes)
        amax = np.abs(ref).max(-1, keepdims=True) * np.sqrt(2)
        assert np.all(np.abs(host(y) - ref) <= HALF[dt] * np.abs(ref) + 2e-5 * amax + 2.0 ** -25)
    major = binding.qk_norm_rope(q, k, norm=norm, q_weight=w[0], q_bias=w[1], k_weight=w[2], k_bias=w[3], eps=1e-5, rope=rope, inv_freq=inv,
                                 positions=ints(pos), axes=ints(axes), head_major=True)
    assert torch.equal(major[0].transpose(0, 1), out[0]) and torch.equal(major[1].transpose(0, 1), out[1])
    if several == 1:                                             # one position: the call without axes
        one = binding.qk_norm_rope(q, k, norm=norm, q_weight=w[0], q_bias=w[1], k_weight=w[2], k_bias=w[3], eps=1e-5, rope=rope, inv_freq=inv,
                                   positions=ints(pos[:, 0]))
        assert torch.equal(one[0], out[0]) and torch.equal(one[1], out[1])


def test_axes_refusals():
    x, f, a, p = torch.zeros(3, 2, 64, device="cuda", dtype=torch.float16), torch.ones(32, device="cuda"), ints(np.zeros(32)), ints(np.zeros((3, 3)))
    ok = dict(rope="half", inv_freq=f, positions=p, axes=a)
    binding.qk_norm_rope(x, x, **ok)
    for bad in (dict(rope="2d"), dict(rope=None), dict(axes=a[:31]), dict(axes=f), dict(positions=p[:, 0].contiguous()), dict(positions=p[:2]),
                dict(positions=ints(np.zeros((3, 9)))), dict(positions=ints(np.zeros((3, 0))))):
        with pytest.raises((ValueError, binding.XsvError)):
            binding.qk_norm_rope(x, x, **{**ok, **bad})


# ------------------------------------------------------------------------------------------------ a server of sequences
class Server:
    """Sequences over a pool, beside their oracle: one Sequence per sequence and head."""

    def __init__(self, n, hkv, d, dtype, pages, width, seed=0, spread=1.0):
        self.n, self.hkv, self.d, self.dt, self.spread = n, hkv, d, DT[dtype], spread
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.pages = binding.page8_pool(pages, hkv, d)
        self.pages.fill_(255)                               # NaN codes and parameters
        self.table = ints(np.full((n, width), -1))
        self.ring, self.state = ints(np.random.default_rng(seed).permutation(pages)), ints([seed % pages, pages, 0, 0])
        self.len = ints(np.zeros(n))
        self.ref = [[orc.Sequence(d) for _ in range(hkv)] for _ in range(n)]
        self.w = 0.5 + torch.rand(hkv, d, device="cuda", generator=self.g)
        self.w[:, ::17] *= 3
        self.mu = 0.5 * torch.randn(hkv, d, device="cuda", generator=self.g)

    def rnd(self, *s):
        return torch.randn(*s, device="cuda", generator=self.g)

    def step(self, new, pad=0, sizes=None):
        """Plans and appends; returns the plan.  sizes: a factor for each token's keys and values."""
        n = int(np.maximum(new, 0).sum())
        plan = binding.page_plan(self.len, ints(new), self.table, self.ring, self.state, n + pad)
        self.len, self.state = plan.total_len, plan.ring_state
        assert plan.ring_state[2] == 0 and plan.ring_state[3] == n
        k = (self.rnd(n + pad, self.hkv, self.d) + self.mu) * self.w * self.spread
        v = self.rnd(n + pad, self.hkv, self.d) * self.spread
        if sizes is not None:
            k, v = (x * torch.tensor(sizes, device="cuda")[:, None, None] for x in (k, v))
        k, v = k.to(self.dt), v.to(self.dt)
        binding.page8_append(self.pages, k, v, plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
        self.note(new, plan, k, v)
        return plan

    def note(self, new, plan, k, v):
        cu = plan.cu_new.cpu().numpy()
        for s in range(self.n):
            for h in range(self.hkv):
                if new[s] < 0:
                    self.ref[s][h] = orc.Sequence(self.d)
                self.ref[s][h].append(host(k[cu[s]:cu[s + 1], h]), host(v[cu[s]:cu[s + 1], h]))

    def check_state(self):
        total, table, rec = self.len.cpu().numpy(), self.table.cpu().numpy(), self.pages.cpu().numpy()
        for s in range(self.n):
            for h in range(self.hkv):
                ref = self.ref[s][h]
                assert ref.n == total[s]
                for b, (k, v) in enumerate(ref.blocks):
                    kc, vc, ks, vs, factor, mean = orc.read_record(rec[table[s, b], h], self.d)
                    m = len(k.codes)
                    assert ks == 2.0 ** k.e and vs == 2.0 ** v.e
                    assert np.array_equal(kc[:m], k.codes) and np.array_equal(vc[:m], v.codes)
                    if m == PAGE:
                        want, f = orc.mean_key(k.codes, k.e)
                        assert np.array_equal(mean, want) and factor == f

    def means(self, s, h):
        return [orc.mean_key(k.codes, k.e) if len(k.codes) == PAGE else None for k, _ in self.ref[s][h].blocks]

    def check_attention(self, plan, new, hq, window=0, scale=None, max_new=None, q=None, **kw):
        n = q.shape[0] if q is not None else int(np.maximum(new, 0).sum())
        q = self.rnd(n, hq, self.d).to(self.dt) if q is None else q
        out = binding.page8_attention(q, self.pages, self.table, plan.cu_new, plan.total_len, int(max(new)) if max_new is None else max_new,
                                      window=window, scale=scale, **kw)
        cu = plan.cu_new.cpu().numpy()
        got, ref, group = host(out), np.zeros(out.shape), hq // self.hkv
        for s in range(self.n):
            for h in range(hq):
                r = self.ref[s][h // group]
                ref[cu[s]:cu[s + 1], h] = orc4.attention(host(q[cu[s]:cu[s + 1], h]), r.k, r.v, scale or self.d ** -0.5, window)
        near(got[:cu[-1]], ref[:cu[-1]], self.dt)
        return out

    def check_selection(self, plan, hq, top, first, recent, q=None):
        """Selects and attends; both against the oracle.  Returns both results."""
        seq, pos, group = plan.token_seq.cpu().numpy(), plan.positions.cpu().numpy(), hq // self.hkv
        q = self.rnd(len(seq), hq, self.d).to(self.dt) if q is None else q
        sel = binding.page8_select(q, self.pages, self.table, plan.token_seq, plan.positions, top, first=first, recent=recent)
        out = binding.page8_attention_selected(q, self.pages, self.table, plan.token_seq, plan.positions, sel)
        got, qh = sel.cpu().numpy(), host(q)
        ref, kv = np.zeros(out.shape), {}
        for t in range(len(seq)):
            for h in range(self.hkv):
                if seq[t] < 0:
                    assert np.all(got[t, h] == -1)
                    continue
                if (seq[t], h) not in kv:
                    r = self.ref[seq[t]][h]
                    kv[seq[t], h] = self.means(seq[t], h), r.k, r.v
                means, k, v = kv[seq[t], h]
                rows = slice(h * group, (h + 1) * group)
                want = orc.select(qh[t, rows], means, pos[t] // PAGE, top, first, recent)
                assert got[t, h].tolist() == want, (t, h)
                at = np.concatenate([np.arange(p * PAGE, min(p * PAGE + PAGE, pos[t] + 1)) for p in want if p >= 0])
                ref[t, rows] = orc.attention(qh[t, rows], k[at], v[at], self.d ** -0.5)
        live = seq >= 0
        near(host(out)[live], ref[live], self.dt)
        return sel, out


# ------------------------------------------------------------------------------------------------ append and read
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d,hkv", [(64, 3), (128, 2), (128, 5)])
def test_append_and_read(dtype, d, hkv):
    sv = Server(4, hkv, d, dtype, pages=60, width=12, seed=5)
    for new in ([1, 64, 63, 200], [1, 1, 1, 0], [62, 0, 65, 1], [1, 129, 300, 63], [70, 2, 0, -1], [5, 64, 1, 10]):
        sv.step(new, pad=3)
        sv.check_state()
        total = sv.len.cpu().numpy()
        # every token, a few that do not exist, in an order of their own
        seq = np.concatenate([np.full(t + 2, s) for s, t in enumerate(total)] + [[-1, 4, 0]])
        pos = np.concatenate([np.arange(-1, t + 1) for t in total] + [[0, 0, 100000]])
        order = np.random.default_rng(1).permutation(len(seq))
        seq, pos = seq[order], pos[order]
        K, V = binding.page8_read(sv.pages, sv.table, sv.len, ints(seq), ints(pos), sv.dt)
        for got, which in ((host(K), "k"), (host(V), "v")):
            vals = [[getattr(sv.ref[s][h], which) for h in range(hkv)] for s in range(4)]
            ref = np.zeros(got.shape)
            for i, (s, p) in enumerate(zip(seq, pos)):
                if 0 <= s < 4 and 0 <= p < total[s]:
                    ref[i] = [vals[s][h][p] for h in range(hkv)]
            assert np.all(np.abs(got - ref) <= (2.0 ** -25 if dtype == "fp16" else 0))


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_scales_grow_with_later_tokens(dtype, d):
    # token by token and in chunks, each a little larger: codes that stand are moved to the new scale, some become subnormal
    sv = Server(3, 2, d, dtype, pages=20, width=4, seed=1, spread=1e-3)
    sv.ref[0][0].append(np.zeros((0, d)), np.zeros((0, d)))
    rng, size = np.random.default_rng(0), 1.0
    for i in range(40):
        new = [1, int(rng.integers(0, 4)), int(rng.integers(1, 6))] if i % 5 else [2, 20, 17]
        size *= float(rng.choice([1.0, 1.0, 1.7, 0.5, 9.0])) if size < 1e5 else 0.01
        sv.step(new, sizes=[size] * sum(new))
        sv.check_state()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_append_at_the_ends_of_the_range(dtype):
    dt = DT[dtype]
    k = torch.zeros(64, 1, 64, device="cuda", dtype=dt)
    k[:, 0, 1] = 7
    k[::2, 0, 2], k[1::2, 0, 2] = 65504 if dtype == "fp16" else 65280, -60000
    if dtype == "bf16":
        k[3, 0, 5], k[4, 0, 6], k[5, 0, 7] = 1e38, -66048, float("inf")       # count as 65504
    else:
        k[5, 0, 7] = float("-inf")
    v = torch.full((64, 1, 64), 1e-6 if dtype == "fp16" else 1e-38, device="cuda").to(dt)
    v[1] = 0
    plan = binding.page_plan(ints([0]), ints([64]), ints([[-1]]), ints([3]), ints([0, 1]), 64)
    pages = binding.page8_pool(4, 1, 64)
    binding.page8_append(pages, k, v, plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
    ref = orc.Sequence(64)
    ref.append(host(k[:, 0]), host(v[:, 0]))
    kc, vc, ks, vs, factor, mean = orc.read_record(pages[3, 0].cpu().numpy(), 64)
    assert np.array_equal(kc, ref.blocks[0][0].codes) and np.array_equal(vc, ref.blocks[0][1].codes) and ks == 256 and vs == 2.0 ** ref.blocks[0][1].e
    want, f = orc.mean_key(kc, 8)
    assert np.array_equal(mean, want) and factor == f
    K, V = binding.page8_read(pages, ints([[3]]), ints([64]), ints([0] * 64), ints(range(64)), dt)
    top = 65504 if dtype == "fp16" else 65536
    assert np.array_equal(host(K)[:, 0], np.clip(ref.k, -top, top)) and K.isfinite().all()
    zero = torch.zeros_like(k)                              # nothing but zeros: no NaN in the mean key
    binding.page8_append(pages, zero, zero, plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
    kc, vc, ks, vs, factor, mean = orc.read_record(pages[3, 0].cpu().numpy(), 64)
    assert not kc.any() and not vc.any() and factor == 0 and not mean.any() and ks == vs == 2.0 ** -80


@pytest.mark.parametrize("d", [64, 128])
def test_append_beside_idle_sequences(d):
    # sequences that bring nothing change nothing, wherever they stand
    n, hkv = 397, 3
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn(n, hkv, d, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    got = []
    for idle in (0, 120):
        pages = binding.page8_pool(12, hkv, d)
        pages.zero_()
        table, state = ints(np.full((3 + idle, 5), -1)), ints([0, 12])
        ring, held = ints(range(12)), ints(np.zeros(3 + idle))
        for new in ([30, 7, 64], [34, 190, 2], [1, 3, 66]):
            m = sum(new)
            plan = binding.page_plan(held, ints(new + [0] * idle), table, ring, state, m)
            held, state = plan.total_len, plan.ring_state
            binding.page8_append(pages, k[:m], v[:m], plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
        got.append(pages)
    assert torch.equal(*got)


def test_append_takes_strided_rows_and_repeats():
    sv = Server(3, 2, 64, "bf16", pages=30, width=8, seed=4)
    sv.step([40, 100, 0])
    for new in ([3, 30, 64], [1, 1, 1]):
        n = sum(new)
        plan = binding.page_plan(sv.len, ints(new), sv.table, sv.ring, sv.state, n)
        both = (4 * sv.rnd(n, 2, 2, 64)).to(sv.dt)          # keys and values side by side in a row; larger than before
        k, v = both[:, 0], both[:, 1]
        args = (plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
        binding.page8_append(sv.pages, k, v, *args)
        state = sv.pages.clone()
        binding.page8_append(sv.pages, k, v, *args)
        assert torch.equal(state, sv.pages)
        sv.note(new, plan, k, v)
        sv.len, sv.state = plan.total_len, plan.ring_state
        sv.check_state()


def test_append_skips_tokens_without_a_place():
    sv = Server(2, 2, 64, "fp16", pages=8, width=4)
    sv.step([10, 70])
    before = sv.pages.clone()
    for idle in (0, 8):
        k = torch.ones(8, 2, 64, device="cuda", dtype=sv.dt)
        for slot, seq, cu, total in (([-1] * 8, [0] * 8, [0, 8, 8], [18, 70]),             # refused
                                     ([5] * 8, [99] * 8, [0, 8, 8], [18, 70]),             # no such sequence
                                     ([64 * 8 + 10 + i for i in range(8)], [0] * 8, [0, 8, 8], [18, 70]),   # no such page
                                     ([20 + i for i in range(8)], [0] * 8, [0, 8, 8], [18, 70]),            # not where the lengths say
                                     ([10 + i for i in range(8)], [0] * 8, [0, 9, 9], [19, 70])):           # more tokens than rows
            binding.page8_append(sv.pages, k, k, ints(slot), ints(seq), ints(cu + cu[-1:] * idle), ints(total + [0] * idle))
            assert torch.equal(before, sv.pages)


# ------------------------------------------------------------------------------------------------ attention
SHAPES = [(64, 3, 3), (64, 8, 2), (128, 4, 4), (128, 8, 1), (128, 20, 4), (64, 12, 1)]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d,hq,hkv", SHAPES)
def test_attention_single_tokens(dtype, d, hq, hkv):
    sv = Server(6, hkv, d, dtype, pages=60, width=16, seed=hq)
    sv.step([0, 62, 63, 64, 200, 700])
    for new in ([1, 1, 1, 1, 1, 1], [1, 1, 0, 1, 1, 1], [1, 1, 1, 1, -1, 1]):
        plan = sv.step(new)
        sv.check_attention(plan, new, hq)
        sv.check_attention(plan, new, hq, window=50)
        sv.check_attention(plan, new, hq, window=130, scale=0.3)


WIDE = 1500           # table rows with room for so much that the kernel for many rows takes what it can


@pytest.mark.parametrize("width", [16, WIDE])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d,hq,hkv", SHAPES)
def test_attention_many_tokens(dtype, d, hq, hkv, width):
    sv = Server(5, hkv, d, dtype, pages=60, width=width, seed=hq + 1)
    for new in ([3, 130, 64, 1, 0], [7, 2, 5, 3, 1], [65, 33, 129, 64, 300]):
        plan = sv.step(new)
        sv.check_attention(plan, new, hq)
        sv.check_attention(plan, new, hq, window=1)
        sv.check_attention(plan, new, hq, window=77)


@pytest.mark.parametrize("new,width", [(1, 8), (40, 8), (40, WIDE)])
@pytest.mark.parametrize("dtype,spread", [("bf16", 1e-12), ("bf16", 1e-3), ("fp16", 1e-3), ("bf16", 300.0), ("fp16", 300.0), ("fp16", 6000.0)])
def test_attention_over_values_of_any_size(new, width, dtype, spread):
    # queries shrink as keys grow, so that the logits stay; the output grows with the values
    sv = Server(2, 2, 64, dtype, pages=20, width=width, seed=3, spread=spread)
    sv.step([300, 70])
    plan = sv.step([new, new])
    scale = None if spread > 1e-6 else 1e12
    q = sv.rnd(2 * new, 4, 64) / (spread if spread > 1e-6 else 8)
    sv.check_attention(plan, [new, new], 4, q=q.to(sv.dt), scale=scale)


@pytest.mark.parametrize("new,width", [(1, 12), (40, 12), (40, WIDE)])
def test_pages_of_very_different_scales(new, width):
    # pages 2^10 apart in both directions: neither the logits' factor nor the values' may come from a neighbour
    sv = Server(1, 2, 128, "bf16", pages=20, width=width, seed=8)
    sizes = np.repeat(2.0 ** np.array([0, -10, 3, -5, 0, -8, 1]), PAGE)
    sv.step([7 * PAGE], sizes=sizes.tolist())
    plan = sv.step([new], sizes=[1.0] * new)
    sv.check_attention(plan, [new], 4, q=(sv.rnd(new, 4, 128) * 0.05).to(sv.dt))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("hq,new", [(12, 4), (12, 10)])     # 48 and 120 query rows a head: both kernels
def test_a_long_sequence_of_values_with_a_mean(d, dtype, hq, new):
    # The weights' roundings, independent over 20 480 tokens, average out against a mean of 3: 2^-11 / sqrt(3 * 20480) of it. What stays is
    # the result's, at most half a step and evenly spread, HALF / sqrt(3) rms; a tenth is left for sums in float32 (320 pages).
    sv = Server(1, 1, d, dtype, pages=330, width=WIDE, seed=d + new)
    for n in (20480, new):
        plan = binding.page_plan(sv.len, ints([n]), sv.table, sv.ring, sv.state, n)
        sv.len, sv.state = plan.total_len, plan.ring_state
        k, v = ((sv.rnd(n, 1, d) + sv.mu) * sv.w).to(sv.dt), (sv.rnd(n, 1, d) + 3).to(sv.dt)
        binding.page8_append(sv.pages, k, v, plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
        sv.note([n], plan, k, v)
    q = sv.rnd(new, hq, d).to(sv.dt)
    out, r = host(binding.page8_attention(q, sv.pages, sv.table, plan.cu_new, plan.total_len, new)), sv.ref[0][0]
    ref = np.stack([orc4.attention(host(q[:, h]), r.k, r.v, d ** -0.5) for h in range(hq)], 1)
    assert np.linalg.norm(out - ref) <= 1.1 * HALF[sv.dt] / np.sqrt(3) * np.linalg.norm(ref)


@pytest.mark.parametrize("new,width", [(1, 8), (3, 8), (60, 8), (60, WIDE)])
def test_attention_past_missing_pages_and_short_rows(new, width):
    sv = Server(2, 2, 64, "bf16", pages=20, width=width, seed=6)
    sv.step([330, 100])
    plan = sv.step([new, new])
    q = sv.rnd(2 * new, 4, 64).to(sv.dt)
    table = sv.table.clone()
    table[0, 1], table[0, 3] = -1, 10 ** 6                  # two pages that are not there
    out = host(binding.page8_attention(q, sv.pages, table, plan.cu_new, plan.total_len, new))
    keep = np.r_[0:64, 128:192, 256:330 + new]
    for i in range(new):
        for h in range(4):
            r = sv.ref[0][h // 2]
            at = keep[keep <= 330 + i]
            ref = orc.attention(host(q[i, h])[None], r.k[at], r.v[at], 1 / 8)[0]
            assert np.linalg.norm(out[i, h] - ref) <= 3 * ATTN[sv.dt] * np.linalg.norm(ref)
    none = host(binding.page8_attention(q, sv.pages, torch.full_like(table, -1), plan.cu_new, plan.total_len, new))
    assert not none.any()
    # a row of the table that is shorter than the sequence: what it does not list is masked, positions stay
    out = host(binding.page8_attention(q, sv.pages, sv.table[:, :2].contiguous(), plan.cu_new, plan.total_len, new))
    for h in range(4):
        r = sv.ref[0][h // 2]
        ref = orc.attention(host(q[0, h])[None], r.k[:128], r.v[:128], 1 / 8)[0]
        assert np.linalg.norm(out[0, h] - ref) <= 3 * ATTN[sv.dt] * np.linalg.norm(ref)


@pytest.mark.parametrize("new,width", [(2, 6), (50, 6), (50, WIDE)])
def test_refused_sequences_and_rows_behind_the_last(new, width):
    sv = Server(3, 2, 64, "fp16", pages=9, width=width, seed=2)
    sv.step([100, 64, 70])
    plan = binding.page_plan(sv.len, ints([new, new, 400]), sv.table, sv.ring, sv.state, 2 * new + 400 + 5)
    assert int(plan.ring_state[2]) == 1
    q = sv.rnd(2 * new + 405, 4, 64).to(sv.dt)
    k = sv.rnd(2 * new + 405, 2, 64).to(sv.dt)
    binding.page8_append(sv.pages, k, k, plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
    out = torch.full_like(q, 7.0)
    binding.page8_attention(q, sv.pages, sv.table, plan.cu_new, plan.total_len, 400, out=out, slot_map=plan.slot_map)
    assert not out[2 * new:2 * new + 400].any() and (out[2 * new + 400:] == 7).all() and out[:2 * new].abs().sum() > 0
    sel = binding.page8_select(q, sv.pages, sv.table, plan.token_seq, plan.positions, 3, slot_map=plan.slot_map)
    assert (sel[2 * new:2 * new + 400] == -1).all() and (sel[2 * new + 400:] == -1).all() and (sel[:2 * new, :, 0] == 0).all()
    out.fill_(7.0)
    binding.page8_attention_selected(q, sv.pages, sv.table, plan.token_seq, plan.positions, sel, out=out)
    assert not out[2 * new:2 * new + 400].any() and (out[2 * new + 400:] == 7).all() and out[:2 * new].abs().sum() > 0


def test_attention_in_the_place_of_the_queries_and_at_a_stride():
    sv = Server(3, 2, 128, "bf16", pages=20, width=WIDE, seed=7)
    for new in ([100, 3, 1], [1, 1, 1], [70, 1, 60]):
        plan = sv.step(new)
        n = sum(new)
        wide = sv.rnd(n, 7, 128).to(sv.dt)
        q = wide[:, 1:5]
        want = sv.check_attention(plan, new, 4, q=q)
        same = q.contiguous()
        binding.page8_attention(same, sv.pages, sv.table, plan.cu_new, plan.total_len, max(new), out=same)
        assert torch.equal(want, same)
        sel = binding.page8_select(q, sv.pages, sv.table, plan.token_seq, plan.positions, 4)
        want = binding.page8_attention_selected(q, sv.pages, sv.table, plan.token_seq, plan.positions, sel)
        same = q.contiguous()
        binding.page8_attention_selected(same, sv.pages, sv.table, plan.token_seq, plan.positions, sel, out=same)
        assert torch.equal(want, same)


# ------------------------------------------------------------------------------------------------ selection
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d,hq,hkv", SHAPES + [(128, 3, 1), (64, 10, 2), (128, 24, 2)])
@pytest.mark.parametrize("top,first,recent", [(4, 1, 2), (1, 0, 1), (9, 2, 3), (30, 0, 2)])
def test_select_and_attend(dtype, d, hq, hkv, top, first, recent):
    sv = Server(5, hkv, d, dtype, pages=90, width=40, seed=hq + top)
    sv.step([0, 62, 64, 700, 1500])
    for new in ([1, 1, 1, 1, 1], [3, 0, 2, 70, 5]):
        plan = sv.step(new, pad=2)
        sv.check_selection(plan, hq, top, first, recent)


@pytest.mark.parametrize("d,hq,hkv,n", [(64, 4, 4, 700), (128, 32, 8, 310), (64, 12, 4, 650)])
def test_select_for_many_tokens(d, hq, hkv, n):
    # enough tokens that a block takes several, some blocks those of two sequences
    sv = Server(4, hkv, d, "bf16", pages=80, width=40, seed=n)
    sv.step([600, 0, 64, 130])
    new = [n // 2 + 1, 3, 0, n - n // 2 - 4]
    plan = sv.step(new, pad=9)
    sv.check_selection(plan, hq, 6, 1, 2)


@pytest.mark.parametrize("d,hq,hkv", [(64, 40, 2), (128, 34, 1), (64, 128, 1), (128, 17, 1)])
def test_large_groups(d, hq, hkv):
    # more query heads to a key/value head than a tile has rows: several tiles of scores and of attention
    sv = Server(3, hkv, d, "bf16", pages=60, width=20, seed=hq)
    sv.step([0, 300, 900])
    for new in ([1, 1, 1], [70, 3, 200]):                   # (one token a block, several)
        plan = sv.step(new, pad=1)
        sv.check_selection(plan, hq, 5, 1, 1)
        sv.check_attention(plan, new, hq)


def test_select_for_many_sequences():
    # a block takes several tokens of as many sequences
    n, hkv, d = 400, 4, 64
    sv = Server(n, hkv, d, "fp16", pages=3 * n, width=4, seed=4)
    sv.step([(37 * i) % 250 for i in range(n)])
    plan = sv.step([1 if i % 7 else 0 for i in range(n)])
    sv.check_selection(plan, 8, 2, 0, 1)


def made_up_pool(pages, hkv, d, g):
    pool = torch.zeros(pages, hkv, 130 * d, dtype=torch.uint8, device="cuda")
    mean = torch.randint(-127, 128, (pages, hkv, d), device="cuda", generator=g, dtype=torch.int8)
    factor = torch.rand(pages, hkv, device="cuda", generator=g)
    pool[..., 128 * d + 32:129 * d + 32] = mean.view(torch.uint8)
    pool[..., 64 * d + 8:64 * d + 12] = factor[..., None].contiguous().view(torch.uint8)
    return pool, mean.cpu().numpy().astype(np.int64), factor.cpu().numpy()


@pytest.mark.parametrize("tokens,width,top", [(1, 32768, 1024), (1, 9000, 3), (160, 1300, 40), (150, 4000, 200)])
def test_select_over_wide_tables(tokens, width, top):
    # more pages than a lane holds scores of, for one token and for several a block; up to the widest table and the longest list
    d, pages, hkv = 64, 3000, 2 if tokens > 1 else 1
    g = torch.Generator(device="cuda").manual_seed(width)
    pool, mean, factor = made_up_pool(pages, hkv, d, g)
    table = torch.randint(0, pages, (1, width), device="cuda", generator=g).to(torch.int32)      # pages appear twice: equal scores
    q = torch.randn(tokens, 2 * hkv, d, device="cuda", generator=g).to(torch.bfloat16)
    positions = [64 * width - 1 - 64 * 7 * i for i in range(tokens)]
    sel = binding.page8_select(q, pool, table, ints([0] * tokens), ints(positions), top, first=1, recent=2).cpu().numpy()
    row, qh = table[0].cpu().numpy(), host(q)
    for t in range(0, tokens, 9):
        for h in range(hkv):
            means = [(mean[p, h], factor[p, h]) for p in row]
            assert sel[t, h].tolist() == orc.select(qh[t, 2 * h:2 * h + 2], means, positions[t] // 64, top, 1, 2)


@pytest.mark.parametrize("hkv,top", [(1, 40), (2, 7), (8, 300)])
def test_select_over_long_sequences(hkv, top):
    # a token whose pages several blocks share
    d, pages = 64, 2500
    g = torch.Generator(device="cuda").manual_seed(top)
    pool = torch.zeros(pages, hkv, 130 * d, dtype=torch.uint8, device="cuda")
    mean = torch.randint(-127, 128, (pages, hkv, d), device="cuda", generator=g, dtype=torch.int8)
    factor = torch.rand(pages, hkv, device="cuda", generator=g)
    mean[1::3] = mean[0]                                    # a third of the pages are alike: equal scores
    factor[1::3] = 0.5
    pool[..., 128 * d + 32:129 * d + 32] = mean.view(torch.uint8)
    pool[..., 64 * d + 8:64 * d + 12] = factor[..., None].contiguous().view(torch.uint8)
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    table = order[None, :2400].contiguous()
    table[0, 100], table[0, 200] = -1, pages                # pages that are not there
    q = torch.randn(3, 4 * hkv, d, device="cuda", generator=g).to(torch.float16)
    positions = [2399 * 64 + 5, 64 * 700, 64 * 90 + 63]
    sel = binding.page8_select(q, pool, table, ints([0, 0, 0]), ints(positions), top, first=2, recent=3).cpu().numpy()
    row, qh, mean, factor = table[0].cpu().numpy(), host(q), mean.cpu().numpy().astype(np.int64), factor.cpu().numpy()
    for t, pos in enumerate(positions):
        for h in range(hkv):
            means = [(mean[p, h], factor[p, h]) if 0 <= p < pages else None for p in row]
            assert sel[t, h].tolist() == orc.select(qh[t, 4 * h:4 * h + 4], means, pos // 64, top, 2, 3)


def test_select_of_equal_and_of_no_scores():
    sv = Server(1, 1, 64, "fp16", pages=30, width=30, seed=1)
    k = torch.ones(20 * 64, 1, 64, device="cuda", dtype=sv.dt)
    plan = binding.page_plan(sv.len, ints([20 * 64]), sv.table, sv.ring, sv.state, 20 * 64)
    binding.page8_append(sv.pages, k, k, plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
    for q in (0.0, 1.0, -1.0, 65504.0):                    # zero, equal and negative scores
        x = torch.full((1, 1, 64), q, device="cuda", dtype=sv.dt)
        sel = binding.page8_select(x, sv.pages, sv.table, ints([0]), ints([1200]), 7, first=1, recent=2)
        assert sel[0, 0].tolist() == [0, 1, 2, 3, 4, 17, 18]
    none = binding.page8_select(torch.ones(3, 1, 64, device="cuda", dtype=sv.dt), sv.pages, sv.table, ints([-1, 1, 0]), ints([5, 5, -1]), 3)
    assert (none == -1).all()
    empty = binding.page8_select(x[:0], sv.pages, sv.table, ints([]), ints([]), 3)
    assert empty.shape == (0, 1, 3)


def test_selections_that_do_not_come_from_select():
    sv = Server(2, 2, 128, "bf16", pages=30, width=12, seed=9)
    sv.step([600, 130])
    plan = sv.step([1, 1])
    q = sv.rnd(2, 4, 128).to(sv.dt)
    lists = [[[0, 3, 3, 5, 9, 10, 12, 40], [9, 2, 5, -1, -1, -1, -1, -1]],     # twice the same, behind the own page, beyond the row
             [[-1, -1, 1, 2, -1, -1, -1, -1], [-1] * 8]]
    seen = [[[0, 3, 5, 9], [9, 5]], [[1, 2], []]]                           # what is above the entry before it, and there
    out = host(binding.page8_attention_selected(q, sv.pages, sv.table, plan.token_seq, plan.positions, ints(lists)))
    pos, ref = [600, 130], np.zeros((2, 4, 128))
    for t in range(2):
        for h in range(2):
            r = sv.ref[t][h]
            at = np.concatenate([np.arange(p * 64, min(p * 64 + 64, pos[t] + 1)) for p in seen[t][h]] + [np.zeros(0, int)]).astype(int)
            ref[t, 2 * h:2 * h + 2] = orc.attention(host(q[t, 2 * h:2 * h + 2]), r.k[at], r.v[at], 128 ** -0.5)
    near(out, ref, sv.dt)
    assert not out[1, 2:].any()
    # all pages selected: the same as attention over everything, up to the order of the additions
    every = ints(np.arange(12)[None, None].repeat(2, 0).repeat(2, 1))
    a = host(binding.page8_attention_selected(q, sv.pages, sv.table, plan.token_seq, plan.positions, every))
    b = host(binding.page8_attention(q, sv.pages, sv.table, plan.cu_new, plan.total_len, 1))
    near(a, b, sv.dt)


# ------------------------------------------------------------------------------------------------ a step as it is used
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp16", 64)])
def test_steps_in_captured_graphs(dtype, d):
    """Plan, rotation by three positions, append, selection and both attentions: eager, and two graphs of the same step
    replayed on two streams at once, each over a pool of its own."""
    hq, hkv, n, dt = 8, 2, 5, DT[dtype]

    def make(seed):
        sv = Server(n, hkv, d, dtype, pages=70, width=16, seed=seed)
        sv.step([130, 64, 700, 1, 300])
        g = torch.Generator(device="cuda").manual_seed(seed)
        x = torch.randn(n, hq + 2 * hkv, d, device="cuda", generator=g).to(dt)
        return sv, x, torch.ones(d, device="cuda", dtype=dt), 10000.0 ** (-torch.arange(d // 2, device="cuda") / (d / 2)), ints(np.arange(d // 2) % 3)

    def step(sv, x, w, inv, axes, state):
        held, ring = state
        plan = binding.page_plan(held, ints_one, sv.table, sv.ring, ring, n)
        three = plan.positions[:, None] + torch.arange(3, device="cuda", dtype=torch.int32)
        q, k = binding.qk_norm_rope(x[:, :hq], x[:, hq:hq + hkv], norm="rms", q_weight=w, k_weight=w, rope="half", inv_freq=inv, positions=three, axes=axes)
        binding.page8_append(sv.pages, k, x[:, hq + hkv:], plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
        full = binding.page8_attention(q, sv.pages, sv.table, plan.cu_new, plan.total_len, 1)
        sel = binding.page8_select(q, sv.pages, sv.table, plan.token_seq, plan.positions, 5)
        part = binding.page8_attention_selected(q, sv.pages, sv.table, plan.token_seq, plan.positions, sel)
        held.copy_(plan.total_len)
        ring.copy_(plan.ring_state)
        return full, sel, part, plan.total_len

    ints_one = ints([1] * n)
    want = []
    for seed in (1, 2):                                     # eager
        sv, x, *rest = make(seed)
        state = [sv.len.clone(), sv.state.clone()]
        for _ in range(66):
            out = step(sv, x, *rest, state)
        want.append([t.clone() for t in out] + [sv.pages])
    graphs = []
    for seed in (1, 2):
        sv, x, *rest = make(seed)
        state = [sv.len.clone(), sv.state.clone()]
        torch.cuda.synchronize()
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=stream):
            out = step(sv, x, *rest, state)
        graphs.append((graph, stream, out, sv, x, rest, state))
    for _ in range(66):
        for graph, stream, *_ in graphs:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for (_, _, out, sv, *_), ref in zip(graphs, want):
        assert all(torch.equal(a, b) for a, b in zip(list(out) + [sv.pages], ref))


def test_calls_repeat_bit_for_bit_and_on_several_streams():
    sv = Server(4, 2, 128, "bf16", pages=60, width=WIDE, seed=12)
    sv.step([900, 300, 64, 0])
    new = [1, 30, 1, 70]
    plan = sv.step(new)
    q = sv.rnd(sum(new), 8, 128).to(sv.dt)
    a = (q, sv.pages, sv.table)

    def all_of(stream=None):
        sel = binding.page8_select(*a, plan.token_seq, plan.positions, 6, stream=stream)
        return (binding.page8_attention(*a, plan.cu_new, plan.total_len, 70, stream=stream), sel,
                binding.page8_attention_selected(*a, plan.token_seq, plan.positions, sel, stream=stream))

    want = all_of()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    got = [all_of(s) for s in streams for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for r in got for x, y in zip(r, want))


def test_pool_beyond_32_bits():
    hkv, d = 8, 128
    n = (1 << 32) // (hkv * 130 * d) + 40                   # the last pages lie behind 4 GB
    pages = binding.page8_pool(n, hkv, d)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(150, hkv, d, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    q = torch.randn(150, 32, d, device="cuda", generator=g).to(torch.bfloat16)
    got = []
    for base in (0, n - 3):
        table, ring = ints([[-1, -1, -1]]), ints([base, base + 1, base + 2])
        plan = binding.page_plan(ints([0]), ints([150]), table, ring, ints([0, 3]), 150)
        binding.page8_append(pages, k, v, plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
        sel = binding.page8_select(q, pages, table, plan.token_seq, plan.positions, 2, first=0, recent=1)
        got.append([binding.page8_attention(q, pages, table, plan.cu_new, plan.total_len, 150), sel,
                    binding.page8_attention_selected(q, pages, table, plan.token_seq, plan.positions, sel),
                    *binding.page8_read(pages, table, plan.total_len, plan.token_seq, plan.positions, torch.bfloat16)])
    assert all(torch.equal(x, y) for x, y in zip(*got)) and got[0][0].isfinite().all()


def test_no_backward():
    sv = Server(1, 1, 64, "fp16", pages=4, width=4)
    plan = sv.step([10])
    q = sv.rnd(10, 1, 64).to(sv.dt).requires_grad_()
    sel = ints(np.zeros((10, 1, 1)))
    for out in (binding.page8_attention(q, sv.pages, sv.table, plan.cu_new, plan.total_len, 10),
                binding.page8_attention_selected(q, sv.pages, sv.table, plan.token_seq, plan.positions, sel)):
        with pytest.raises(RuntimeError):
            out.sum().backward()


def test_binding_refusals():
    sv = Server(2, 2, 64, "fp16", pages=6, width=4)
    plan = sv.step([10, 3])
    q, k = sv.rnd(13, 4, 64).to(sv.dt), sv.rnd(13, 2, 64).to(sv.dt)
    P, t = sv.pages, sv.table
    seq, pos, cu, total, slot = plan.token_seq, plan.positions, plan.cu_new, plan.total_len, plan.slot_map
    sel = binding.page8_select(q, P, t, seq, pos, 3)
    bad = [lambda: binding.page8_append(P, k.float(), k, slot, seq, cu, total), lambda: binding.page8_append(P, k, k.to(torch.bfloat16), slot, seq, cu, total),
           lambda: binding.page8_append(P[..., :-1], k, k, slot, seq, cu, total), lambda: binding.page8_append(P, k[:, :1], k, slot, seq, cu, total),
           lambda: binding.page8_append(P, k, k, slot[:12], seq, cu, total), lambda: binding.page8_append(P, k, k, slot, seq, cu[:2], total),
           lambda: binding.page8_append(P.transpose(0, 1), k, k, slot, seq, cu, total), lambda: binding.page8_read(P, t, total, seq, pos, torch.float32),
           lambda: binding.page8_read(P, t, total, seq, pos, "fp16"), lambda: binding.page8_read(P, t, total, seq[:3], pos, torch.float16),
           lambda: binding.page8_attention(q[..., :32], P, t, cu, total, 10), lambda: binding.page8_attention(q, P, t, cu, total, 10, out=q[:5]),
           lambda: binding.page8_attention(q, P, t[:1], cu, total, 10), lambda: binding.page8_attention(q, P, t, cu, total, 10, slot_map=slot[:5]),
           lambda: binding.page8_select(q, P, t, seq[:5], pos, 3), lambda: binding.page8_select(q, P, t, seq, pos, 0), lambda: binding.page8_select(q, P, t, seq, pos, 1 << 20),
           lambda: binding.page8_select(q, P, t.long(), seq, pos, 3), lambda: binding.page8_select(q, P, t, seq, pos, 3, slot_map=slot[:5]),
           lambda: binding.page8_attention_selected(q, P, t, seq, pos, sel[:5]), lambda: binding.page8_attention_selected(q, P, t, seq, pos, sel.long())]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: binding.page8_attention(q[:, :3], P, t, cu, total, 10), lambda: binding.page8_attention(q, P, t, cu, total, 10, scale=-1.0),
                 lambda: binding.page8_select(q, P, t, seq, pos, 3, first=2), lambda: binding.page8_select(q, P, t, seq, pos, 3, recent=0),
                 lambda: binding.page8_attention_selected(q, P, t, seq, pos, sel, scale=float("nan")),
                 lambda: binding.page8_attention_selected(q, P, t, seq, pos, sel[..., :0].contiguous())):
        with pytest.raises(binding.XsvError):
            call()
