"""The operators over a shared pool of 4-bit pages against the float64 oracle, on the GPU.

Tolerances.  A result that is rounded once to the output type is off by at most half a step, eps / 2 relative (2^-11 for
fp16, 2^-8 for bf16).
  norm and rotation: besides that, float32 arithmetic on a row whose largest element is A: the sums over 128 channels, a
    rounding each, give at most 128 * 2^-24 relative on the mean and half of it on the root, the rotation, its angle and the
    products another 8 * 2^-24: below 2e-5 * A in all.
  append, read: codes and parameters are those of the oracle, bit for bit; a value read back is rounded once to float32 and
    once to the output type.
  attention: P s and q s are rounded to fp16 (2^-11 relative each).  P s weighs codes up to 15 s, about four times a value's
    own spread: 4 * 2^-11 of the output's noise-like magnitude.  q s moves a logit by sqrt(d) independent terms of
    2^-11 |q| 15 s / sqrt(d), about 2^-11 * 4 at unit variances: as much again.  With the output's own half step that is
    2^-8 + 8 * 2^-11 = 8e-3 of the 2-norm for bf16, 5e-3 for fp16, over all rows; a single row may be three times that.
"""
import numpy as np
import pytest
import torch

from oracle import page_oracle as orc
from paper_2602_21780_b200 import binding

pytestmark = pytest.mark.gpu

PAGE = 64
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
ATTN = {torch.float16: 5e-3, torch.bfloat16: 8e-3}
DT = {"fp16": torch.float16, "bf16": torch.bfloat16}


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def host(t):
    return t.double().cpu().numpy()


# ------------------------------------------------------------------------------------------------ norm and rotation
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d,hq,hkv,n", [(64, 3, 3, 1), (128, 8, 1, 1), (64, 16, 16, 261), (128, 20, 4, 700), (64, 5, 1, 7)])
@pytest.mark.parametrize("norm,rope,rotary", [("rms", "half", None), ("layer", "2d", None), (None, "pairs", None), ("rms", "half", 32),
                                              ("layer", "pairs", 24), ("layer", None, None), (None, None, None)])
def test_norm_rope(dtype, d, hq, hkv, n, norm, rope, rotary):
    dt = DT[dtype]
    g = torch.Generator(device="cuda").manual_seed(d + n)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    # rows of a fused projection with a gap behind them
    fused = (rnd(n, (hq + 2 * hkv) * d + 8) * (0.1 + 3 * torch.rand(n, 1, device="cuda", generator=g)) + 0.3).to(dt)
    q, k, v = (fused[:, a * d:b * d].view(n, b - a, d) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
    w = [None] * 4
    if norm:
        w = [(1 + 0.3 * rnd(d)).to(dt), None, (1 + 0.3 * rnd(d)).to(dt), (0.2 * rnd(d)).to(dt)]
    r = d if rotary is None else rotary
    inv, pos = None, None
    if rope == "2d":
        inv, pos = 100.0 ** (-torch.arange(d // 4, device="cuda") / (d / 4)), ints(np.random.default_rng(n).integers(0, 40, (n, 2)))
    elif rope:
        inv = 10000.0 ** (-torch.arange(r // 2, device="cuda") / (r / 2))
        pos = ints(np.random.default_rng(n).integers(-5, 2_000_000, n))
    for head_major in (False, True):
        out = binding.qk_norm_rope(q, k, v, norm=norm, q_weight=w[0], q_bias=w[1], k_weight=w[2], k_bias=w[3], eps=1e-5, rope=rope,
                                   inv_freq=inv, positions=pos, head_major=head_major)
        if head_major:
            assert out[0].shape == (hq, n, d) and all(t.is_contiguous() for t in out)
            out = [t.transpose(0, 1) for t in out]
        assert torch.equal(out[2], v)
        for x, y, ww, bb in ((q, out[0], w[0], w[1]), (k, out[1], w[2], w[3])):
            ref = orc.norm_rope(host(x), norm, None if ww is None else host(ww), None if bb is None else host(bb), 1e-5, rope, r,
                                None if inv is None else host(inv), None if pos is None else pos.cpu().numpy())
            amax = np.abs(ref).max(-1, keepdims=True) * np.sqrt(2)
            assert np.all(np.abs(host(y) - ref) <= HALF[dt] * np.abs(ref) + 2e-5 * amax + 2.0 ** -25)
    two = binding.qk_norm_rope(q, k, norm=norm, q_weight=w[0], q_bias=w[1], k_weight=w[2], k_bias=w[3], eps=1e-5, rope=rope,
                               inv_freq=inv, positions=pos)
    assert len(two) == 2 and torch.equal(two[0], out[0]) and torch.equal(two[1], out[1])


def test_norm_rope_of_no_tokens_and_of_a_zero_row():
    z = torch.zeros(0, 2, 64, device="cuda", dtype=torch.float16)
    assert binding.qk_norm_rope(z, z, z, norm="rms")[0].shape == (0, 2, 64)
    z = torch.zeros(2, 2, 64, device="cuda", dtype=torch.float16)
    assert not any(t.any() for t in binding.qk_norm_rope(z, z, norm="layer", eps=1e-6))


# ------------------------------------------------------------------------------------------------ plan
def plan_inputs(n, seed, width=40, spare=30, extra_pages=0):
    rng = np.random.default_rng(seed)
    cached = np.where(rng.random(n) < 0.2, 0, rng.integers(0, 1500, n))
    new = rng.choice([-1, 0, 1, 1, 1, 5, 64, 200], n)
    have = -(-cached // PAGE)
    pages = int(have.sum()) + spare + extra_pages
    order = rng.permutation(pages)
    table, used = np.full((n, width), -1), 0
    for s in range(n):
        table[s, :have[s]] = order[used:used + have[s]]
        used += have[s]
    ring, head = np.full(pages, -1), int(rng.integers(0, pages))
    for i, p in enumerate(order[used:]):
        ring[(head + i) % pages] = p
    return cached, new, table.astype(np.int32), ring.astype(np.int32), [head, pages - used]


def check_plan(cached, new, table, ring, state, most):
    t, r = ints(table), ints(ring)
    dev = [ints(cached), ints(new), t, r, ints(state)]
    got = binding.page_plan(*dev, most)
    first = [x.clone() for x in (t, r, *got)]
    again = binding.page_plan(*dev, most)                   # the same inputs: the same outputs
    assert all(torch.equal(a, b) for a, b in zip(first, (t, r, *again)))
    table, ring = table.copy(), ring.copy()
    want = orc.plan(cached, new, table, ring, state, most)
    assert np.array_equal(t.cpu().numpy(), table) and np.array_equal(r.cpu().numpy(), ring)
    for name, w in zip(("ring_state", "cu_new", "total_len", "slot_map", "token_seq", "positions"), want):
        assert np.array_equal(getattr(got, name).cpu().numpy(), w), name
    return got


@pytest.mark.parametrize("n", [1, 2, 33, 512, 513, 1300, 8192])
def test_plan_against_the_oracle(n):
    c = plan_inputs(n, n, spare=5 * n + 3)
    tokens = int(np.maximum(c[1], 0).sum())
    check_plan(*c, tokens)
    check_plan(*c, tokens + 2500)                           # rows behind the last token


def test_plan_refuses_what_does_not_fit():
    for seed in range(6):
        cached, new, table, ring, state = plan_inputs(50, seed, width=24, spare=6)
        tokens = int(np.maximum(new, 0).sum())
        got = check_plan(cached, new, table, ring, state, tokens)          # too few pages
        assert got.ring_state[2] > 0
        check_plan(cached, new, table, ring, state, tokens // 2)           # too few places for tokens
        check_plan(cached, new, table, ring, state, 0)
    cached, new, table, ring, state = plan_inputs(20, 9, spare=100)
    check_plan(cached, new, np.ascontiguousarray(table[:, :24]), ring, state, int(np.maximum(new, 0).sum()))   # rows that are full


def test_plan_of_ended_and_waiting_sequences_only():
    cached, new, table, ring, state = plan_inputs(30, 3)
    check_plan(cached, np.full(30, -1), table, ring, state, 4)
    check_plan(cached, np.zeros(30, int), table, ring, state, 4)


# ------------------------------------------------------------------------------------------------ a server of sequences
class Server:
    """Sequences over a pool, beside their oracle: one Sequence per sequence and head."""

    def __init__(self, n, hkv, d, dtype, pages, width, seed=0, spread=1.0):
        self.n, self.hkv, self.d, self.dt, self.spread = n, hkv, d, DT[dtype], spread
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.pages, self.tail = binding.page_pool(pages, n, hkv, d, self.dt)
        self.pages.fill_(255)                               # NaN parameters, largest codes
        self.tail.fill_(float("nan"))
        self.table = ints(np.full((n, width), -1))
        self.ring, self.state = ints(np.random.default_rng(seed).permutation(pages)), ints([seed % pages, pages, 0, 0])
        self.len = ints(np.zeros(n))
        self.ref = [[orc.Sequence(d) for _ in range(hkv)] for _ in range(n)]
        # per-channel weights and offsets: a few channels large
        self.w = 0.5 + torch.rand(hkv, d, device="cuda", generator=self.g)
        self.w[:, ::17] *= 3
        self.mu = 0.5 * torch.randn(hkv, d, device="cuda", generator=self.g)

    def rnd(self, *s):
        return torch.randn(*s, device="cuda", generator=self.g)

    def step(self, new, pad=0):
        """Plans and appends; returns the plan."""
        n = int(np.maximum(new, 0).sum())
        plan = binding.page_plan(self.len, ints(new), self.table, self.ring, self.state, n + pad)
        self.len, self.state = plan.total_len, plan.ring_state
        assert plan.ring_state[2] == 0 and plan.ring_state[3] == n
        k = ((self.rnd(n + pad, self.hkv, self.d) + self.mu) * self.w * self.spread).to(self.dt)
        v = (self.rnd(n + pad, self.hkv, self.d) * self.spread).to(self.dt)
        binding.page_append(self.pages, self.tail, k, v, plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
        cu = plan.cu_new.cpu().numpy()
        for s in range(self.n):
            for h in range(self.hkv):
                if new[s] < 0:
                    self.ref[s][h] = orc.Sequence(self.d)
                self.ref[s][h].append(host(k[cu[s]:cu[s + 1], h]), host(v[cu[s]:cu[s + 1], h]))
        return plan

    def check_state(self):
        total, table = self.len.cpu().numpy(), self.table.cpu().numpy()
        rec = self.pages.cpu().numpy()
        for s in range(self.n):
            for h in range(self.hkv):
                ref = self.ref[s][h]
                assert len(ref.k) == total[s]
                for b in range(-(-int(total[s]) // PAGE)):
                    k, v = orc.read_record(rec[table[s, b], h], self.d)
                    m = min(PAGE, int(total[s]) - b * PAGE)
                    assert np.array_equal(v[:m], ref.v[b * PAGE:b * PAGE + m])
                    if m == PAGE:
                        assert np.array_equal(k, ref.k[b * PAGE:b * PAGE + PAGE])
                    else:
                        assert np.array_equal(host(self.tail[s, b % 2, h, :m]), ref.k[b * PAGE:])

    def check_attention(self, plan, new, hq, window=0, scale=None, max_new=None, q=None, **kw):
        n = q.shape[0] if q is not None else int(np.maximum(new, 0).sum())
        q = self.rnd(n, hq, self.d).to(self.dt) if q is None else q
        out = binding.page_attention(q, self.pages, self.tail, self.table, plan.cu_new, plan.total_len,
                                     int(max(new)) if max_new is None else max_new, window=window, scale=scale, **kw)
        cu = plan.cu_new.cpu().numpy()
        got, ref, group = host(out), np.zeros(out.shape), hq // self.hkv
        for s in range(self.n):
            for h in range(hq):
                r = self.ref[s][h // group]
                ref[cu[s]:cu[s + 1], h] = orc.attention(host(q[cu[s]:cu[s + 1], h]), r.k, r.v, scale or self.d ** -0.5, window)
        live = slice(0, cu[-1])
        err, size = np.linalg.norm(got[live] - ref[live], axis=-1), np.linalg.norm(ref[live], axis=-1)
        tol = ATTN[self.dt]
        assert np.all(np.isfinite(got[live]))
        assert np.linalg.norm(err) <= tol * np.linalg.norm(size)
        assert np.all(err <= 3 * tol * size + 1e-6)
        return out


# ------------------------------------------------------------------------------------------------ append and read
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d,hkv", [(64, 3), (128, 2)])
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
        K, V = binding.page_read(sv.pages, sv.tail, sv.table, sv.len, ints(seq), ints(pos))
        for got, which in ((host(K), "k"), (host(V), "v")):
            ref = np.zeros(got.shape)
            for i, (s, p) in enumerate(zip(seq, pos)):
                if 0 <= s < 4 and 0 <= p < total[s]:
                    ref[i] = [getattr(sv.ref[s][h], which)[p] for h in range(hkv)]
            assert np.all(np.abs(got - ref) <= HALF[sv.dt] * np.abs(ref) * 1.001 + 2.0 ** -25)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("spread", [1e-4, 3000.0])
def test_append_at_the_ends_of_the_range(dtype, spread):
    sv = Server(2, 1, 64, dtype, pages=9, width=4, seed=2, spread=spread)
    sv.step([130, 64])
    sv.check_state()
    # constant rows, zeros, and the largest values
    k = torch.zeros(64, 1, 64, device="cuda", dtype=sv.dt)
    k[:, 0, 1] = 7
    k[::2, 0, 2], k[1::2, 0, 2] = 65504 if dtype == "fp16" else 65280, -60000
    plan = binding.page_plan(ints([0]), ints([64]), ints([[-1]]), ints([3]), ints([0, 1]), 64)
    pages, tail = binding.page_pool(4, 1, 1, 64, sv.dt)
    binding.page_append(pages, tail, k, k, plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
    ref = orc.Sequence(64)
    ref.append(host(k[:, 0]), host(k[:, 0]))
    got_k, got_v = orc.read_record(pages[3, 0].cpu().numpy(), 64)
    assert np.array_equal(got_k, ref.k) and np.array_equal(got_v, ref.v)


def test_append_takes_strided_rows_and_repeats():
    sv = Server(3, 2, 64, "bf16", pages=30, width=8, seed=4)
    sv.step([40, 100, 0])
    new = [3, 30, 64]
    plan = binding.page_plan(sv.len, ints(new), sv.table, sv.ring, sv.state, 97)
    both = sv.rnd(97, 2, 2, 64).to(sv.dt)                   # keys and values side by side in a row
    k, v = both[:, 0], both[:, 1]
    args = (plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
    binding.page_append(sv.pages, sv.tail, k, v, *args)
    state = sv.pages.clone(), sv.tail.clone()
    binding.page_append(sv.pages, sv.tail, k, v, *args)
    assert torch.equal(state[0], sv.pages) and torch.equal(state[1].view(torch.int16), sv.tail.view(torch.int16))
    cu = plan.cu_new.cpu().numpy()
    for s in range(3):
        for h in range(2):
            sv.ref[s][h].append(host(k[cu[s]:cu[s + 1], h]), host(v[cu[s]:cu[s + 1], h]))
    sv.len = plan.total_len
    sv.check_state()


def test_append_skips_tokens_without_a_place():
    sv = Server(2, 2, 64, "fp16", pages=8, width=4)
    sv.step([10, 70])
    before = sv.pages.clone(), sv.tail.clone()
    k = torch.ones(8, 2, 64, device="cuda", dtype=sv.dt)
    for slot, seq, cu, total in (([-1] * 8, [0] * 8, [0, 8, 8], [18, 70]),             # refused
                                 ([5] * 8, [7] * 8, [0, 8, 8], [18, 70]),              # no such sequence
                                 ([64 * 8 + 10 + i for i in range(8)], [0] * 8, [0, 8, 8], [18, 70]),   # no such page
                                 ([20 + i for i in range(8)], [0] * 8, [0, 8, 8], [18, 70]),            # not where the lengths say
                                 ([10 + i for i in range(8)], [0] * 8, [0, 9, 9], [19, 70])):           # more tokens than rows
        binding.page_append(sv.pages, sv.tail, k, k, ints(slot), ints(seq), ints(cu), ints(total))
        assert torch.equal(before[0], sv.pages) and torch.equal(before[1].view(torch.int16), sv.tail.view(torch.int16))


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


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d,hq,hkv", SHAPES)
def test_attention_many_tokens(dtype, d, hq, hkv):
    sv = Server(5, hkv, d, dtype, pages=60, width=16, seed=hq + 1)
    for new in ([3, 130, 64, 1, 0], [7, 2, 5, 3, 1], [65, 33, 129, 64, 300]):
        plan = sv.step(new)
        sv.check_attention(plan, new, hq)
        sv.check_attention(plan, new, hq, window=1)
        sv.check_attention(plan, new, hq, window=77)


@pytest.mark.parametrize("spread", [1e-3, 1.0, 300.0])
def test_attention_over_values_of_any_size(spread):
    # queries shrink as keys grow, so that the logits stay; the output grows with the values
    sv = Server(2, 2, 64, "bf16", pages=20, width=8, seed=3, spread=spread)
    plan = sv.step([300, 70])
    new = [1, 1]
    plan = sv.step(new)
    sv.check_attention(plan, new, 4, q=(sv.rnd(2, 4, 64) / spread).to(sv.dt))


def test_attention_when_value_scales_grow_along_the_sequence():
    sv = Server(1, 1, 64, "fp16", pages=20, width=16, seed=3)
    for i in range(6):
        sv.spread = 1.0
        n = 64
        plan = binding.page_plan(sv.len, ints([n]), sv.table, sv.ring, sv.state, n)
        sv.len, sv.state = plan.total_len, plan.ring_state
        k, v = sv.rnd(n, 1, 64).to(sv.dt), (sv.rnd(n, 1, 64) * 10.0 ** (i - 3)).to(sv.dt)
        binding.page_append(sv.pages, sv.tail, k, v, plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
        sv.ref[0][0].append(host(k[:, 0]), host(v[:, 0]))
    sv.check_attention(plan, [64], 2)


def test_attention_with_queries_of_any_size():
    sv = Server(2, 1, 128, "bf16", pages=20, width=8, seed=8)
    sv.step([150, 70])
    plan = sv.step([1, 1])
    q = sv.rnd(2, 4, 128)
    q[0, 1] = 0                                             # uniform over everything
    q[1, 0] *= 1e-20
    q[1, 1] *= 40                                           # one key takes it all
    sv.check_attention(plan, [1, 1], 4, q=q.to(sv.dt))


def test_attention_padded_batch_and_strided_queries():
    sv = Server(3, 2, 64, "bf16", pages=30, width=10, seed=6)
    sv.step([100, 0, 500])
    new = [2, 0, 1]
    plan = sv.step(new, pad=4)
    wide = sv.rnd(7, 3, 4, 64).to(sv.dt)
    out = torch.full((7, 4, 64), 7.0, device="cuda", dtype=sv.dt)
    got = sv.check_attention(plan, new, 4, q=wide[:, 1], out=out, max_new=50)
    assert got is out and bool((out[3:] == 7).all())        # rows behind the last sequence


def test_attention_of_sequences_that_hold_nothing():
    sv = Server(2, 1, 64, "fp16", pages=8, width=4)
    sv.step([70, 0])
    # a sequence that the plan refused: it brings rows but holds nothing
    q = sv.rnd(3, 2, 64).to(sv.dt)
    out = binding.page_attention(q, sv.pages, sv.tail, sv.table, ints([0, 0, 3]), ints([70, 0]), 3)
    assert not out.any()
    # more rows than tokens: the first rows lie before the sequence's start
    out = binding.page_attention(q, sv.pages, sv.tail, sv.table, ints([0, 3, 3]), ints([1, 0]), 3)
    assert not out[:2].any()
    # pages that do not exist are masked: only the second page's tokens are seen
    table = sv.table.clone()
    table[0, 0] = 8
    out = binding.page_attention(q[:1], sv.pages, sv.tail, table, ints([0, 1, 1]), ints([70, 0]), 1)
    r = sv.ref[0][0]
    ref = orc.attention(host(q[0]), r.k[64:], r.v[64:], 64 ** -0.5)
    ref[:-1] = orc.attention(host(q[0, :1]), r.k[64:], r.v[64:], 64 ** -0.5)
    assert np.abs(host(out[0, 0]) - ref[0]).max() <= 0.02 * np.abs(ref[0]).max()
    table[0, :] = -1
    assert not binding.page_attention(q[:1], sv.pages, sv.tail, table, ints([0, 1, 1]), ints([70, 0]), 1).any()


def test_attention_many_short_sequences_and_the_largest_count():
    n = 700
    sv = Server(n, 1, 64, "bf16", pages=n, width=1, seed=11)
    new = (np.arange(n) % 63 + 1).tolist()
    plan = sv.step(new)
    sv.check_attention(plan, new, 2)
    new = [1 if i % 3 else 0 for i in range(n)]
    plan = sv.step(new)
    sv.check_attention(plan, new, 2)


def test_pages_behind_four_gigabytes():
    # a pool of 4.6 GB; the sequence's pages lie at its end
    d, hkv, pages = 128, 8, 63000
    sv = Server(1, hkv, d, "bf16", pages=8, width=4, seed=1)
    sv.pages, _ = binding.page_pool(pages, 1, hkv, d, sv.dt)
    sv.ring, sv.state = ints(np.arange(pages)[::-1].copy()), ints([0, 5])
    plan = sv.step([190])
    assert int(sv.table[0, 0]) == pages - 1
    plan = sv.step([1])
    sv.check_attention(plan, [1], 16)
    seq, pos = ints([0, 0]), ints([0, 190])
    K, V = binding.page_read(sv.pages, sv.tail, sv.table, sv.len, seq, pos)
    for i, p in enumerate((0, 190)):
        ref = np.stack([sv.ref[0][h].v[p] for h in range(hkv)])
        assert np.all(np.abs(host(V[i]) - ref) <= HALF[sv.dt] * np.abs(ref) * 1.001)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d,hq,hkv", [(64, 4, 4), (64, 12, 1), (128, 8, 2), (128, 5, 5)])
def test_attention_of_a_long_chunk_shared_by_many_blocks(dtype, d, hq, hkv):
    sv = Server(1, hkv, d, dtype, pages=70, width=64, seed=d + hq)
    sv.step([3001])
    for new in (700, 65, 258):
        plan = sv.step([new])
        sv.check_attention(plan, [new], hq)
        sv.check_attention(plan, [new], hq, window=500)


def test_attention_of_decoding_and_prompt_sequences_in_one_call():
    sv = Server(6, 2, 64, "bf16", pages=80, width=24, seed=21)
    sv.step([500, 3, 64, 1000, 0, 0])
    for new in ([1, 400, 2, 90, 0, 1], [1, 1, 300, 1, 20, 17], [33, 16, 17, 1, 64, 65]):
        plan = sv.step(new, pad=5)
        n = sum(new) + 5
        out = torch.full((n, 8, 64), 7.0, device="cuda", dtype=sv.dt)
        q = sv.rnd(n, 8, 64).to(sv.dt)
        sv.check_attention(plan, new, 8, q=q, out=out, max_new=500)
        assert bool((out[-5:] == 7).all())
        again = binding.page_attention(q, sv.pages, sv.tail, sv.table, plan.cu_new, plan.total_len, max(new))
        assert torch.equal(again[:-5], out[:-5])             # the bound on the new tokens changes nothing


def test_long_chunks_of_sequences_that_hold_nothing_or_miss_pages():
    sv = Server(2, 1, 64, "fp16", pages=8, width=6)
    plan = sv.step([300, 0])
    q = sv.rnd(300, 2, 64).to(sv.dt)
    out = binding.page_attention(q, sv.pages, sv.tail, sv.table, ints([0, 0, 300]), ints([300, 0]), 300)
    assert not out.any()
    out = binding.page_attention(q, sv.pages, sv.tail, sv.table, ints([0, 300, 300]), ints([100, 0]), 300)
    assert not out[:200].any() and out[200:].any()
    # without its second page, a sequence sees the others; rows before it see the first alone
    table = sv.table.clone()
    table[0, 1] = -1
    out = host(binding.page_attention(q, sv.pages, sv.tail, table, plan.cu_new, plan.total_len, 300))
    r = sv.ref[0][0]
    qh, keep = host(q), np.r_[0:64, 128:300]
    for i in (0, 63, 64, 127, 128, 299):
        at = keep[keep <= i]
        w = np.exp(r.k[at] @ qh[i].T / 8 - (r.k[at] @ qh[i].T / 8).max(0))
        ref = (w / w.sum(0)).T @ r.v[at]
        assert np.abs(out[i] - ref).max() <= 0.02 * np.abs(ref).max()
    table[0, :] = 8
    assert not binding.page_attention(q, sv.pages, sv.tail, table, plan.cu_new, plan.total_len, 300).any()


def test_long_chunks_repeat_bit_for_bit_and_from_a_graph():
    sv = Server(3, 2, 128, "bf16", pages=80, width=40, seed=13)
    sv.step([2000, 30, 0])
    new = [300, 200, 90]
    plan = sv.step(new)
    q = sv.rnd(590, 8, 128).to(sv.dt)
    want = sv.check_attention(plan, new, 8, q=q)
    for _ in range(3):
        assert torch.equal(want, binding.page_attention(q, sv.pages, sv.tail, sv.table, plan.cu_new, plan.total_len, 300))
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        out = binding.page_attention(q, sv.pages, sv.tail, sv.table, plan.cu_new, plan.total_len, 300)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want, out)


def test_append_of_many_decoding_sequences_beside_a_prompt():
    n = 41
    sv = Server(n, 2, 128, "bf16", pages=140, width=40, seed=15)
    sv.step((np.arange(n) * 7 % 130).tolist())
    for _ in range(3):
        sv.step([600 if s == 20 else 1 + s % 9 for s in range(n)], pad=2)
        sv.check_state()
    sv.step([1] * n)
    sv.check_state()


def test_append_keeps_a_value_that_is_not_finite_from_its_neighbours():
    for dtype in ("fp16", "bf16"):
        for bad in (float("inf"), float("-inf"), float("nan")):
            dt = DT[dtype]
            k = torch.randn(64, 1, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(dt)
            ref = orc.Sequence(64)
            ref.append(host(k[:, 0]), host(k[:, 0]))
            k[5, 0, 7] = bad
            plan = binding.page_plan(ints([0]), ints([64]), ints([[-1]]), ints([0]), ints([0, 1]), 64)
            pages, tail = binding.page_pool(1, 1, 1, 64, dt)
            binding.page_append(pages, tail, k, k, plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
            got_k, got_v = orc.read_record(pages[0, 0].cpu().numpy(), 64)
            channels, tokens = np.arange(64) != 7, np.arange(64) != 5
            assert np.array_equal(got_k[:, channels], ref.k[:, channels]) and np.array_equal(got_v[tokens], ref.v[tokens])


# ------------------------------------------------------------------------------------------------ together
def test_a_serving_step_captured_and_replayed_on_other_streams():
    # norm + rotation -> append -> attention of a decode step, captured; lengths live on the device, so one graph serves
    # every step.  Two graphs (two layers) with workspaces of their own replay on two streams at once.
    n, hq, hkv, d, dt = 5, 8, 2, 64, torch.bfloat16
    eager = [Server(n, hkv, d, "bf16", pages=40, width=8, seed=s) for s in (1, 2)]
    for sv in eager:
        sv.step([10, 63, 64, 127, 200])
    inv = 10000.0 ** (-torch.arange(d // 2, device="cuda") / (d / 2))
    w = torch.ones(d, device="cuda", dtype=dt)
    graphs = []
    for sv in eager:
        st = dict(len=sv.len.clone(), new=ints([1] * n), table=sv.table.clone(), ring=sv.ring.clone(), state=sv.state.clone(),
                  pages=sv.pages.clone(), tail=sv.tail.clone(), q=torch.empty(n, hq, d, device="cuda", dtype=dt),
                  k=torch.empty(n, hkv, d, device="cuda", dtype=dt), v=torch.empty(n, hkv, d, device="cuda", dtype=dt))

        def step(st=st):
            p = binding.page_plan(st["len"], st["new"], st["table"], st["ring"], st["state"], n)
            q, k, v = binding.qk_norm_rope(st["q"], st["k"], st["v"], norm="rms", q_weight=w, k_weight=w, rope="half", inv_freq=inv,
                                           positions=p.positions)
            binding.page_append(st["pages"], st["tail"], k, v, p.slot_map, p.token_seq, p.cu_new, p.total_len)
            out = binding.page_attention(q, st["pages"], st["tail"], st["table"], p.cu_new, p.total_len, 1)
            return out, p, k, v

        for t in (st["q"], st["k"], st["v"]):
            t.normal_()
        keep = {k: v.clone() for k, v in st.items()}
        step()                                              # warm-up; its effects are undone
        for k in st:
            st[k].copy_(keep[k])
        torch.cuda.synchronize()
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=side):
            out, p, k, v = step()
            st["len"].copy_(p.total_len)                    # the next replay goes on from here
            st["state"].copy_(p.ring_state)
        graphs.append((graph, torch.cuda.Stream(), st, out, p, k, v, step))
    for _ in range(4):
        for graph, stream, st, *_ in graphs:
            for t in (st["q"], st["k"], st["v"]):
                t.normal_()
        torch.cuda.synchronize()
        for graph, stream, *_ in graphs:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for sv, (graph, stream, st, out, p, k, v, step) in zip(eager, graphs):
            cu = p.cu_new.cpu().numpy()
            for s in range(n):
                for h in range(hkv):
                    sv.ref[s][h].append(host(k[s:s + 1, h]), host(v[s:s + 1, h]))
            sv.pages, sv.tail, sv.table, sv.len = st["pages"], st["tail"], st["table"], st["len"]
            sv.check_state()
            q, _, _ = binding.qk_norm_rope(st["q"], st["k"], st["v"], norm="rms", q_weight=w, k_weight=w, rope="half", inv_freq=inv,
                                           positions=p.positions)
            again = sv.check_attention(p, [1] * n, hq, q=q)
            assert torch.equal(again, out) and cu[-1] == n


def test_norm_and_rotation_feed_a_cache_step():
    # a frame of 5 special tokens and 6 x 6 patches: layer norm, rotation by row and column, then the streaming step
    from oracle import xsv_oracle
    n, h, d, dt = 41, 4, 64, torch.float16
    g = torch.Generator(device="cuda").manual_seed(3)
    at = (torch.arange(n, device="cuda") - 5).clamp(min=-1)
    pos = torch.stack([at // 6 + 1, at % 6 + 1], -1)
    pos = torch.where(at[:, None] < 0, torch.zeros_like(pos), pos).to(torch.int32).contiguous()
    inv = 100.0 ** (-torch.arange(d // 4, device="cuda") / (d / 4))
    cache, ref = binding.Cache(1, h, d, 82, 4), xsv_oracle.LayerCache(h, d, 82, 4)
    for _ in range(4):
        q, k, v = (torch.randn(n, h, d, device="cuda", generator=g).to(dt) for _ in range(3))
        Q, K, V = binding.qk_norm_rope(q, k, v, norm="layer", eps=1e-5, rope="2d", inv_freq=inv, positions=pos, head_major=True)
        want = orc.norm_rope(host(q), "layer", None, None, 1e-5, "2d", d, host(inv), pos.cpu().numpy()).transpose(1, 0, 2)
        assert np.all(np.abs(host(Q) - want) <= HALF[dt] * np.abs(want) + 2e-5 * np.abs(want).max())
        out = torch.empty_like(Q)
        cache.step(0, Q, K, V, out)
        o = ref.step(*(t.float().cpu().numpy() for t in (Q, K, V)))
        assert np.abs(out.float().cpu().numpy() - o).max() <= 1e-2 * np.abs(o).max()      # the step's own tolerance
    cache.destroy()


def test_calls_on_a_given_stream():
    sv = Server(2, 2, 64, "fp16", pages=12, width=6, seed=9)
    plan = sv.step([100, 30])
    plan = sv.step([1, 1])
    q = sv.rnd(2, 4, 64).to(sv.dt)
    want = sv.check_attention(plan, [1, 1], 4, q=q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = binding.page_attention(q, sv.pages, sv.tail, sv.table, plan.cu_new, plan.total_len, 1, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def test_results_repeat_bit_for_bit():
    sv = Server(3, 2, 128, "bf16", pages=200, width=100, seed=12)
    sv.step([5000, 900, 3])
    plan = sv.step([1, 1, 1])
    q = sv.rnd(3, 16, 128).to(sv.dt)
    a = sv.check_attention(plan, [1, 1, 1], 16, q=q)
    for _ in range(5):
        assert torch.equal(a, binding.page_attention(q, sv.pages, sv.tail, sv.table, plan.cu_new, plan.total_len, 1))


def test_binding_checks_shapes_and_types():
    sv = Server(2, 2, 64, "fp16", pages=8, width=4)
    plan = sv.step([10, 70])
    q = sv.rnd(80, 4, 64).to(sv.dt)
    ok = dict(Q=q, pages=sv.pages, k_tail=sv.tail, block_table=sv.table, cu_new=plan.cu_new, total_len=plan.total_len, max_new=70)
    binding.page_attention(**ok)
    for bad in (dict(Q=q.float()), dict(Q=q.to(torch.bfloat16)), dict(Q=q[:, :, :32]), dict(Q=q.transpose(0, 1)), dict(Q=q.cpu()),
                dict(block_table=sv.table.long()), dict(block_table=sv.table[:1]), dict(cu_new=plan.cu_new[:2]),
                dict(pages=sv.pages[..., :72]), dict(out=torch.empty_like(q)[1:])):
        with pytest.raises(ValueError):
            binding.page_attention(**{**ok, **bad})
    with pytest.raises(binding.XsvError):
        binding.page_attention(**{**ok, "scale": -1.0})
    with pytest.raises(binding.XsvError):
        binding.page_attention(**{**ok, "window": -1})
    with pytest.raises(ValueError):
        binding.qk_norm_rope(q, q[:5])
    with pytest.raises(ValueError):
        binding.qk_norm_rope(q, q, rope="half")
    with pytest.raises(ValueError):
        binding.page_append(sv.pages, sv.tail, q[:, :2], q[:, :2], plan.slot_map[:3], plan.token_seq, plan.cu_new, plan.total_len)
    with pytest.raises(ValueError):
        binding.page_plan(sv.len, ints([1, 1]).long(), sv.table, sv.ring, sv.state, 3)
