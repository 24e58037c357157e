"""The operators over a shared pool of 4-bit pages where their descriptions end: hand-overs between the kernels' roles, the
ends of the number range, refused sequences, bounds that are too small, scales that underflow."""
import numpy as np
import pytest
import torch

from oracle import page_oracle as orc
from paper_2602_21780_b200 import binding
from tests.test_gpu_page_ops import ATTN, DT, HALF, PAGE, Server, host, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,hq,hkv,new", [(64, 3, 3, 101), (128, 4, 2, 60)])
def test_long_units_without_a_second_query_tile(d, hq, hkv, new):
    # at most 128 query rows a head over more pages than the ring of stages holds twice: the warp that would serve the second
    # tile passes every stage's phases and releases its share of them; a longer chunk beside it changes between both kinds
    sv = Server(3, hkv, d, "bf16", pages=170, width=64, seed=d + new)
    sv.step([3003, 2500, 1100])
    for step in ([new, 0, 0], [new, 400, new + 1], [0, new, 300]):
        plan = sv.step(step)
        sv.check_attention(plan, step, hq)


def top_rows(n, hkv, d, dt, g):
    """Keys and values whose groups span to the largest finite values: 0, 65504 and both ends, where outward rounding alone
    would let the last code stand for more than float16 holds."""
    top = torch.finfo(torch.float16).max
    k = torch.randn(n, hkv, d, device="cuda", generator=g)
    k[::2, :, 3], k[1::2, :, 3] = 0, top
    k[::2, :, 9], k[1::2, :, 9] = top, -top
    v = torch.rand(n, hkv, d, device="cuda", generator=g)
    low = torch.tensor([0.0, -top, -60000.0, 0.5 * top], device="cuda")[torch.arange(n, device="cuda") % 4]
    v = low[:, None, None] + (top - low[:, None, None]) * v
    v[:, :, ::64], v[:, :, 1::64] = low[:, None, None], top
    return k.to(dt), v.clamp(-top, top).to(dt)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_values_at_the_top_of_the_range_stay_finite(dtype, d):
    # 200 tokens by 2 heads: few rows a head (1 new token) and many (90); queries so small that the logits stay near 1
    sv = Server(1, 2, d, dtype, pages=6, width=4, seed=d)
    k, v = top_rows(200, 2, d, sv.dt, sv.g)
    plan = binding.page_plan(sv.len, ints([200]), sv.table, sv.ring, sv.state, 200)
    binding.page_append(sv.pages, sv.tail, k, v, plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
    sv.len = plan.total_len
    for h in range(2):
        sv.ref[0][h].append(host(k[:, h]), host(v[:, h]))
    sv.check_state()
    K, V = binding.page_read(sv.pages, sv.tail, sv.table, sv.len, ints([0] * 200), ints(np.arange(200)))
    for got, which in ((host(K), "k"), (host(V), "v")):
        ref = np.stack([getattr(r, which) for r in sv.ref[0]], 1)
        assert np.all(np.abs(got - ref) <= HALF[sv.dt] * np.abs(ref) * 1.001 + 2.0 ** -25)
    q = (sv.rnd(90, 4, d) * 1e-5).to(sv.dt)
    for new in (1, 90):
        fake = plan._replace(cu_new=ints([0, new]))
        sv.check_attention(fake, [new], 4, q=q[:new].contiguous(), scale=1.0)


@pytest.mark.parametrize("new", [1, 6])
def test_a_mean_of_the_largest_values_stays_finite(new):
    # 60 values of 65504; one token's weight is 1, the others' lie just above the middle between two float16 numbers next to
    # 1/2, so that all of them are rounded up by nearly 2^-11: the mean leaves float16 unless it is brought back.  12 query
    # heads by 6 tokens go to the kernel for many rows, 12 rows to the one for few.
    sv = Server(1, 1, 64, "fp16", pages=2, width=1)
    top = 65504.0
    k = torch.zeros(60, 1, 64, device="cuda", dtype=sv.dt)
    k[0, 0, 0] = 1
    v = torch.full((60, 1, 64), top, device="cuda", dtype=sv.dt)
    plan = binding.page_plan(sv.len, ints([60]), sv.table, sv.ring, sv.state, 60)
    binding.page_append(sv.pages, sv.tail, k, v, plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
    q = torch.zeros(new, 12, 64, device="cuda", dtype=sv.dt)
    q[:, :, 0] = 1
    scale = (1 - np.log2(1 + 1.05 * 2.0 ** -11)) / np.log2(np.e)
    out = host(binding.page_attention(q, sv.pages, sv.tail, sv.table, ints([0, new]), plan.total_len, new, scale=float(scale)))
    assert np.all(np.abs(out - top) <= 2.0 ** -11 * top)        # exactly 65504 in real arithmetic


@pytest.mark.parametrize("d,hq,hkv", [(64, 4, 4), (128, 8, 2)])
def test_any_bound_on_the_new_tokens_gives_the_same_rows(d, hq, hkv):
    # it chooses kernels and tiles; the rows attended and their positions come from the lengths
    sv = Server(4, hkv, d, "bf16", pages=60, width=14, seed=31)
    sv.step([70, 0, 300, 5])
    new = [3, 150, 1, 70]
    plan = sv.step(new)
    for bound in (1, 2, 20, 149, 224, 1 << 30):
        sv.check_attention(plan, new, hq, max_new=bound)
    sv.check_attention(plan, new, hq, max_new=1, window=40)
    one = Server(1, hkv, d, "bf16", pages=20, width=14, seed=32)          # a single sequence, whose kernel a loose bound changes
    one.step([200])
    plan = one.step([2])
    q = one.rnd(90, hq, d).to(one.dt)
    for bound in (1, 2, 90):
        out = torch.full((90, hq, d), 7.0, device="cuda", dtype=one.dt)
        one.check_attention(plan, [2], hq, max_new=bound, q=q, out=out)
        assert bool((out[2:] == 7).all())


@pytest.mark.parametrize("d,hq,hkv", [(64, 4, 2), (128, 8, 1)])
def test_rows_of_refused_sequences_that_hold_tokens_are_zero(d, hq, hkv):
    # refused for each of the three reasons, with few rows a head and with many, beside sequences that are served
    held = [60, 128, 250, 64, 190]
    for new, pages_left, width, room in (([3, 1, 2, 1, 1], 1, 5, 99),               # 1 takes the page; 3 needs one and is refused
                                         ([100, 90, 130, 300, 2], 4, 9, 999),       # 0, 1 take two each; 2, 3 refused
                                         ([1, 70, 1, 200, 2], 9, 4, 999),           # 3's row of the table is full, 2 and 4 fit
                                         ([1, 5, 90, 80, 20], 9, 9, 150)):          # 3 and 4 are cut by max_tokens
        sv = Server(5, hkv, d, "bf16", pages=40, width=width, seed=sum(new))
        sv.step(held)
        state = sv.state.clone()
        state[1] = pages_left
        plan = binding.page_plan(sv.len, ints(new), sv.table, sv.ring, state, room)
        cu, total = plan.cu_new.cpu().numpy(), plan.total_len.cpu().numpy()
        slot = plan.slot_map.cpu().numpy()
        n = int(cu[-1])
        refused = [s for s in range(5) if total[s] == held[s]]
        assert refused == {1: [3], 4: [2, 3], 9: [3] if width == 4 else [3, 4]}[pages_left] and int(plan.ring_state[2]) == len(refused)
        k, v = (sv.rnd(n, hkv, d).to(sv.dt) for _ in range(2))
        binding.page_append(sv.pages, sv.tail, k, v, plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)
        for s in range(5):
            if s not in refused:
                for h in range(hkv):
                    sv.ref[s][h].append(host(k[cu[s]:cu[s + 1], h]), host(v[cu[s]:cu[s + 1], h]))
        q = sv.rnd(n, hq, d).to(sv.dt)
        out = host(binding.page_attention(q, sv.pages, sv.tail, sv.table, plan.cu_new, plan.total_len, max(new), slot_map=plan.slot_map))
        for s in range(5):
            rows = slice(cu[s], cu[s + 1])
            if s in refused:
                assert np.all(slot[rows] == -1) and not out[rows].any()
                continue
            for h in range(hq):
                r = sv.ref[s][h // (hq // hkv)]
                ref = orc.attention(host(q[rows, h]), r.k, r.v, d ** -0.5)
                assert np.linalg.norm(out[rows, h] - ref) <= 3 * ATTN[sv.dt] * np.linalg.norm(ref)
        # a plan that refused nothing: the slots change nothing, bit for bit
    sv = Server(3, hkv, d, "fp16", pages=40, width=9, seed=1)
    plan = sv.step([100, 2, 70])
    q = sv.rnd(172, hq, d).to(sv.dt)
    a = sv.check_attention(plan, [100, 2, 70], hq, q=q)
    assert torch.equal(a, sv.check_attention(plan, [100, 2, 70], hq, q=q, slot_map=plan.slot_map))
    with pytest.raises(ValueError, match="fewer tokens"):
        binding.page_attention(q, sv.pages, sv.tail, sv.table, plan.cu_new, plan.total_len, 100, slot_map=plan.slot_map[:171])


@pytest.mark.parametrize("new", [1, 100])
def test_logits_too_small_for_float32_weigh_all_tokens_alike(new):
    # scale * |q| below the smallest float32: the factor of a masked place's -infinity must not become 0
    sv = Server(2, 1, 64, "bf16", pages=20, width=8, seed=new)
    sv.step([90, 30])
    plan = sv.step([new, new])
    q = (sv.rnd(2 * new, 2, 64) * 1e-20).to(sv.dt)
    sv.check_attention(plan, [new, new], 2, q=q, scale=1e-30)
    sv.check_attention(plan, [new, new], 2, q=q, scale=1e-30, window=33)
    sv.check_attention(plan, [new, new], 2, q=(q.float() * 1e-18).to(sv.dt))          # the smallest normal queries


def test_a_backward_pass_is_refused_and_not_silently_empty():
    sv = Server(1, 2, 64, "bf16", pages=4, width=2)
    plan = sv.step([5])
    q, k, v = (sv.rnd(5, h, 64).to(sv.dt) for h in (4, 2, 2))
    w = torch.nn.Parameter(torch.ones(64, device="cuda", dtype=sv.dt))
    att = (sv.pages, sv.tail, sv.table, plan.cu_new, plan.total_len, 5)
    with torch.no_grad():
        plain = binding.qk_norm_rope(q, k, v, norm="rms", q_weight=w, k_weight=w)
    assert not any(t.requires_grad for t in plain)
    out = binding.qk_norm_rope(q, k, v, norm="rms", q_weight=w, k_weight=w)
    assert all(torch.equal(a, b) for a, b in zip(plain, out))
    with pytest.raises(RuntimeError, match="qk_norm_rope is not implemented"):
        out[0].float().sum().backward()
    assert w.grad is None
    q.requires_grad_()
    out = binding.page_attention(q, *att)
    with pytest.raises(RuntimeError, match="page_attention is not implemented"):
        out.float().sum().backward()
    with torch.inference_mode():
        assert torch.equal(binding.page_attention(q, *att), out)
    k.requires_grad_()
    binding.page_append(sv.pages, sv.tail, k, v, plan.slot_map, plan.token_seq, plan.cu_new, plan.total_len)      # stores numbers
    assert not binding.page_attention(q.detach(), *att).requires_grad


@pytest.mark.parametrize("new", [6, 30])
def test_append_reads_one_slot_a_page(new):
    # the first new token's slot in each page decides for all of the sequence's tokens there (few of them: a warp; more: a block)
    def grown(change):
        sv = Server(1, 2, 64, "bf16", pages=4, width=3, seed=new)
        sv.step([64 - new // 2])
        plan = binding.page_plan(sv.len, ints([new]), sv.table, sv.ring, sv.state, new)
        slots = plan.slot_map.clone()
        for i in change:
            slots[i] = -1
        k, v = (torch.randn(new, 2, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(sv.dt) for _ in range(2))
        before = sv.pages.clone(), sv.tail.clone()
        binding.page_append(sv.pages, sv.tail, k, v, slots, plan.token_seq, plan.cu_new, plan.total_len)
        old, fresh = (int(x) for x in sv.table[0, :2])
        same = [torch.equal(sv.pages[p], before[0][p]) for p in (old, fresh)]
        return sv.pages, sv.tail.view(torch.int16), same

    whole = grown([])
    assert whole[2] == [False, False]
    inside = grown([1, new // 2 + 1])                       # inside both pages' tokens: nothing changes
    assert torch.equal(whole[0], inside[0]) and torch.equal(whole[1], inside[1])
    assert grown([0])[2] == [True, False]                   # the first page's tokens are skipped, the second's are not
    assert grown([new // 2])[2] == [False, True]
    assert grown([0, new // 2])[2] == [True, True]


def test_an_argument_without_a_truth_value_is_refused():
    q = torch.zeros(3, 2, 64, device="cuda", dtype=torch.float16)
    with pytest.raises(ValueError, match="true or false"):
        binding.qk_norm_rope(q, q, head_major=np.zeros(2))


def served(d, hq, hkv, held, new, seed):
    """A step over random tokens; the oracle is not grown."""
    sv = Server(len(held), hkv, d, "bf16", pages=sum(held + new) // 64 + 3 * len(held), width=80, seed=seed)
    for m in (held, new):
        n = sum(m)
        plan = binding.page_plan(sv.len, ints(m), sv.table, sv.ring, sv.state, n)
        sv.len, sv.state = plan.total_len, plan.ring_state
        binding.page_append(sv.pages, sv.tail, sv.rnd(n, hkv, d).to(sv.dt), sv.rnd(n, hkv, d).to(sv.dt), plan.slot_map, plan.token_seq,
                            plan.cu_new, plan.total_len)
    q = sv.rnd(sum(new), hq, d).to(sv.dt)

    def attend(**kw):
        return binding.page_attention(kw.pop("q", q), sv.pages, sv.tail, sv.table, plan.cu_new, plan.total_len, max(new), **kw)
    return q, attend


JOBS = [(64, 16, 16, [3000], [1374]), (128, 32, 8, [2000] * 4, [1] * 4), (128, 8, 2, [1500, 100, 900], [300, 1, 65]), (64, 8, 2, [700, 1], [2, 90])]


def test_calls_on_several_streams_at_once():
    jobs = [served(*job, seed=i)[1] for i, job in enumerate(JOBS)]
    want = [attend() for attend in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(10):
        got = [attend(stream=s) for _ in range(2) for attend, s in zip(jobs, streams)]
        torch.cuda.synchronize()
        for a, b in zip(got, want + want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("job", JOBS)
def test_results_in_the_place_of_the_queries(job):
    q, attend = served(*job, seed=7)
    want = attend()
    own = q.clone()
    assert attend(q=own, out=own) is own and torch.equal(own, want)


@pytest.mark.parametrize("window", [0, 150])
@pytest.mark.parametrize("d,hq,hkv", [(64, 4, 2), (128, 8, 1)])
def test_tokens_beyond_a_table_row_are_masked(d, hq, hkv, window):
    # the lengths say more than the row has pages for: positions stay, the tokens behind the row are not seen
    sv = Server(3, hkv, d, "bf16", pages=40, width=12, seed=3)
    sv.step([500, 320, 100])
    for new in ([1, 3, 1], [120, 2, 60]):
        plan = sv.step(new)
        q = sv.rnd(sum(new), hq, d).to(sv.dt)
        total, cu = plan.total_len.cpu().numpy(), plan.cu_new.cpu().numpy()
        for width in (5, 2):
            out = host(binding.page_attention(q, sv.pages, sv.tail, sv.table[:, :width].contiguous(), plan.cu_new, plan.total_len, max(new), window=window))
            for s in range(3):
                seen = min(int(total[s]), width * PAGE)
                for h in range(hq):
                    r = sv.ref[s][h // (hq // hkv)]
                    for i in range(0, new[s], 7):
                        at = int(total[s]) - new[s] + i
                        lo, hi = max(0, at - window + 1) if window else 0, min(at + 1, seen)
                        ref = np.zeros(d)
                        if lo < hi:
                            ref = orc.attention(host(q[cu[s] + i, h])[None], r.k[lo:hi], r.v[lo:hi], d ** -0.5)[0]
                        assert np.linalg.norm(out[cu[s] + i, h] - ref) <= 3 * ATTN[sv.dt] * np.linalg.norm(ref)
