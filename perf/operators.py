"""Operators that serve many ragged sequences from one pool of 4-bit pages: what each is asked to do, its plain form
in elementary torch operations, and the sizes it is used at.

  norm_rope   queries and keys normalised per head and rotated by position in one pass, laid out for the attention
  plan        block tables, slot map, positions and free list of a step, from the sequences' lengths
  append      new keys and values quantised into pages of 64 tokens, and the touched pages read back as values
  attention   ragged causal attention (grouped heads, one or many new tokens per sequence) over the pages

A page record holds 64 tokens of one key/value head, 72 * head_dim bytes:
  [0, 32 d)    4-bit key codes, bytes [d/16 k][8 g][4 j][4 m][4 b]: the low nibble is token 16 m + g, the high one
               token 16 m + 8 + g, channel 32 (k/2) + 8 j + 4 (k%2) + 2 (b%2) + b/2
  [32 d, 64 d) 4-bit value codes, bytes [4 k][d/64 c][8 g][4 j][4 m][4 b]: token 16 k + 8 (b%2) + 2 j + b/2, the low
               nibble channel 64 c + 8 g + 2 m, the high one the channel after it
  [64 d, 72 d) float16: key scale [d], key offset [d] (per channel), value scale [d/64][8 g][8 i], value offset the
               same (per token 8 i + g and 64 channels)
A value is code * scale + offset; offset = the group's minimum rounded down to float16, scale = (maximum - offset) / 15
rounded up to float16 (1 where that is 0), code = nearest-even of (x - offset) / scale.  The keys of a sequence's last,
unfilled page stay as they came, in k_tail[sequence][page % 2][head][64][d]; its values are in the page.
"""
import math

import numpy as np
import torch

own = False

PAGE = 64


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token of one sequence: the decode step's smallest launch, where latency is all there is
        dict(name="norm_rope one token", op="norm_rope", tokens=1, q_heads=32, kv_heads=8, d=128, norm="rms", rope="half",
             far=30000, head_major=False, dtype="bf16"),
        # one video frame of the streaming configuration: 5 special tokens and 37 x 37 patches, rotated by row and column
        dict(name="norm_rope frame 1374", op="norm_rope", tokens=1374, q_heads=16, kv_heads=16, d=64, norm="layer",
             rope="2d", far=37, head_major=True, dtype="bf16"),
        # a long prompt
        dict(name="norm_rope prompt 8191", op="norm_rope", tokens=8191, q_heads=32, kv_heads=8, d=128, norm="rms",
             rope="half", far=131072, head_major=False, dtype="fp16"),
        # a few sequences, one token each
        dict(name="plan 7 sequences", op="plan", seqs=7, cached_lo=100, cached_hi=3000, new_lo=1, new_hi=1, mixed=False),
        # a busy server's step: decoding sequences, prompts, finished and idle ones
        dict(name="plan 1021 mixed", op="plan", seqs=1021, cached_lo=0, cached_hi=16000, new_lo=1, new_hi=700, mixed=True),
        # decode step of a batch
        dict(name="append decode 256", op="append", seqs=256, cached_lo=65, cached_hi=4000, new_lo=1, new_hi=1,
             kv_heads=8, d=128, dtype="bf16"),
        # prompts of ragged lengths, continued from page boundaries
        dict(name="append prompts 5", op="append", seqs=5, cached_lo=0, cached_hi=2048, new_lo=1500, new_hi=9001,
             kv_heads=8, d=64, dtype="fp16"),
        # one short sequence, one token: latency
        dict(name="attention one of 261", op="attention", seqs=1, total_lo=261, total_hi=261, new_lo=1, new_hi=1,
             q_heads=16, kv_heads=16, d=64, window=0, dtype="fp16"),
        # a decode batch of ragged lengths, grouped heads
        dict(name="attention decode 64", op="attention", seqs=64, total_lo=900, total_hi=16000, new_lo=1, new_hi=1,
             q_heads=32, kv_heads=8, d=128, window=0, dtype="bf16"),
        # one very long sequence, four tokens at once (drafted tokens being verified)
        dict(name="attention 4 of 200001", op="attention", seqs=1, total_lo=200001, total_hi=200001, new_lo=4, new_hi=4,
             q_heads=32, kv_heads=8, d=128, window=0, dtype="bf16"),
        # a whole video frame over a cache of the streaming configuration's budget
        dict(name="attention frame on 21984", op="attention", seqs=1, total_lo=23358, total_hi=23358, new_lo=1374,
             new_hi=1374, q_heads=16, kv_heads=16, d=64, window=0, dtype="bf16"),
        # ragged chunks of prompts, grouped heads
        dict(name="attention chunks 6", op="attention", seqs=6, total_lo=2100, total_hi=9000, new_lo=300, new_hi=2047,
             q_heads=32, kv_heads=8, d=128, window=0, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_rope", "plan", "append", "attention", "attention"])
    dtype = rng.choice(["bf16", "fp16"])
    q_heads, kv_heads, d = rng.choice([(32, 8, 128), (16, 16, 64), (8, 1, 128), (20, 4, 128), (12, 4, 64), (5, 5, 64)])
    if op == "norm_rope":
        rope = rng.choice(["half", "pairs", "2d"])
        return dict(op=op, tokens=_log(rng, 1, 8000), q_heads=q_heads, kv_heads=kv_heads, d=d,
                    norm=rng.choice(["rms", "layer", "none"]), rope=rope, far=37 if rope == "2d" else _log(rng, 100, 1000000),
                    head_major=rng.random() < 0.5, dtype=dtype)
    if op == "plan":
        return dict(op=op, seqs=_log(rng, 1, 1000), cached_lo=0, cached_hi=_log(rng, 50, 16000), new_lo=1,
                    new_hi=_log(rng, 1, 600), mixed=rng.random() < 0.7)
    if op == "append":
        if rng.random() < 0.5:
            return dict(op=op, seqs=_log(rng, 1, 256), cached_lo=0, cached_hi=_log(rng, 50, 3000), new_lo=1,
                        new_hi=rng.choice([1, 1, 2, 5]), kv_heads=kv_heads, d=d, dtype=dtype)
        return dict(op=op, seqs=rng.randint(1, 6), cached_lo=0, cached_hi=_log(rng, 64, 2000), new_lo=70,
                    new_hi=_log(rng, 100, 6000), kv_heads=kv_heads, d=d, dtype=dtype)
    window = 0 if rng.random() < 0.7 else _log(rng, 100, 5000)
    if rng.random() < 0.6:
        seqs = _log(rng, 1, 64)
        most = 15000 if seqs > 8 else 90000 // seqs
        hi = _log(rng, 60, most)
        return dict(op=op, seqs=seqs, total_lo=max(8, hi // rng.choice([1, 3, 10])), total_hi=hi, new_lo=1,
                    new_hi=rng.choice([1, 1, 1, 2, 7]), q_heads=q_heads, kv_heads=kv_heads, d=d, window=window, dtype=dtype)
    seqs = rng.randint(1, 5)
    new_hi = _log(rng, 40, 1300)
    return dict(op=op, seqs=seqs, total_lo=new_hi, total_hi=new_hi + _log(rng, 10, 6000), new_lo=max(1, new_hi // 4),
                new_hi=new_hi, q_heads=q_heads, kv_heads=kv_heads, d=d, window=window, dtype=dtype)


# A case's ragged lengths are a function of the case alone, spread over [lo, hi]; a single sequence has the upper end.
def _spread(i, n, lo, hi):
    if n == 1 or hi <= lo:
        return hi
    return lo + (((i * 2654435761 + 40503) % 4294967296) * (hi - lo + 1) >> 32)


def _lengths(case):
    """Per sequence: (tokens cached before the call, new tokens)."""
    n = case["seqs"]
    new = [_spread(3 * i + 1, n, case["new_lo"], case["new_hi"]) for i in range(n)]
    if case["op"] == "attention":
        total = [_spread(i, n, case["total_lo"], case["total_hi"]) for i in range(n)]
        return [max(0, t - m) for t, m in zip(total, new)], new
    cached = [_spread(i, n, case["cached_lo"], case["cached_hi"]) for i in range(n)]
    if case["op"] == "append":          # chunks of a prompt end at a page's end; a few decoded tokens start anywhere
        cached = [c // PAGE * PAGE if m > PAGE else c for c, m in zip(cached, new)]
    if case["op"] == "plan" and case["mixed"]:
        # four of five sequences decode one token, some are finished (-1), some wait (0), the rest bring prompts
        new = [m if i % 7 == 0 else -1 if i % 11 == 5 else 0 if i % 13 == 3 else 1 for i, m in enumerate(new)]
    return cached, new


def _visible(case):
    """Query-key pairs that the mask leaves, over all sequences."""
    pairs = 0
    for c, m in zip(*_lengths(case)):
        for i in (range(m) if m < 4096 else ()):
            seen = c + i + 1
            pairs += min(seen, case["window"]) if case["window"] else seen
    return pairs


def work(case):
    op = case["op"]
    if op == "norm_rope":
        rows = case["tokens"] * (case["q_heads"] + 2 * case["kv_heads"])
        return dict(bytes=4 * rows * case["d"] + 4 * case["tokens"], flops=10 * rows * case["d"])
    cached, new = _lengths(case)
    if op == "plan":
        tokens = sum(max(0, m) for m in new)
        blocks = sum(-(-(c + m) // PAGE) - -(-c // PAGE) if m > 0 else -(-c // PAGE) if m < 0 else 0
                     for c, m in zip(cached, new))
        return dict(bytes=12 * tokens + 16 * case["seqs"] + 8 * blocks, flops=4 * tokens)
    hkv, d = case["kv_heads"], case["d"]
    if op == "append":
        tokens = sum(new)
        back = sum(c + m - c // PAGE * PAGE for c, m in zip(cached, new))
        # new rows read, pages written, the touched pages read back and written out as values
        return dict(bytes=hkv * d * (4 * tokens + 72 * tokens // PAGE + 72 * back // PAGE + 4 * back),
                    flops=hkv * d * (8 * tokens + 4 * back))
    held = 0
    for c, m in zip(cached, new):
        first = max(0, c - case["window"] + 1) if case["window"] else 0
        held += (c + m - first) * 72 * d // PAGE + (c + m) % PAGE * 2 * d
    return dict(bytes=hkv * held + 4 * sum(new) * case["q_heads"] * d,
                flops=4 * _visible(case) * case["q_heads"] * d)


# ------------------------------------------------------------------------------------------------ inputs
def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _down(x):
    """The largest float16 not above x (float64 or float32)."""
    h = x.clamp(-65504, 65504).to(torch.float16)
    i = h.view(torch.int16).to(torch.int32)
    below = torch.where(h > 0, i - 1, torch.where(h == 0, torch.full_like(i, -32767), i + 1))
    return torch.where(h.to(x.dtype) > x, below.to(torch.int16).view(torch.float16), h)


def _quantise(x, dim):
    """4-bit codes along dim: (codes, scale, offset), the last two as float16 with dim kept."""
    x = x.clamp(-65504, 65504)
    z = _down(x.amin(dim, keepdim=True))
    s = -_down(-((x.amax(dim, keepdim=True) - z.to(x.dtype)) / 15))
    s = torch.where(s == 0, torch.ones_like(s), s)
    return ((x - z.to(x.dtype)) / s.to(x.dtype)).round().clamp(0, 15), s, z


def _pack(kc, ks, kz, vc, vs, vz):
    """Records [..., 72 d] of codes [..., 64, d], key parameters [..., d] and value parameters [..., d/64, 64]."""
    lead, d = kc.shape[:-2], kc.shape[-1]
    b = len(lead)
    at = lambda *o: tuple(range(b)) + tuple(b + i for i in o)  # noqa: E731
    k = kc.to(torch.uint8).view(*lead, 4, 2, 8, d // 32, 4, 2, 2, 2).permute(at(3, 5, 2, 4, 0, 7, 6, 1))
    v = vc.to(torch.uint8).view(*lead, 4, 2, 4, 2, d // 64, 8, 4, 2).permute(at(0, 4, 5, 2, 6, 3, 1, 7))
    vs, vz = (t.view(*lead, d // 64, 8, 8).transpose(-1, -2) for t in (vs, vz))
    parts = [(t[..., 0] | t[..., 1] << 4).reshape(*lead, 32 * d) for t in (k, v)]
    params = torch.cat([t.reshape(*lead, -1) for t in (ks, kz, vs, vz)], -1)
    return torch.cat(parts + [params.view(torch.uint8)], -1)


def _cache(case, cached, held, g):
    """Pool, tails and block table of sequences with `cached` tokens in place, in tables that have room for `held`."""
    hkv, d, dt, n = case["kv_heads"], case["d"], _dt(case), case["seqs"]
    blocks = [-(-h // PAGE) for h in held]
    width, pages = max(1, max(blocks)), sum(blocks) + 3
    # keys after their norm: per-channel weights, a few channels large, offsets of their own; values plain
    m = 0.6 + 0.8 * torch.rand(hkv, 1, d, device="cuda", generator=g)
    m[:, :, torch.randint(0, d, (3,), device="cuda", generator=g)] *= 3
    mu = 0.5 * torch.randn(hkv, 1, d, device="cuda", generator=g)
    pool = torch.empty(pages, hkv, 72 * d, dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 25) // (hkv * PAGE * d))
    for p in range(0, pages, step):
        c = min(step, pages - p)
        k = ((torch.randn(c, hkv, PAGE, d, device="cuda", generator=g) + mu) * m).to(dt).float()
        v = torch.randn(c, hkv, PAGE, d, device="cuda", generator=g).to(dt).float()
        kc, ks, kz = _quantise(k, -2)
        vc, vs, vz = _quantise(v.view(c, hkv, PAGE, d // 64, 64), -1)
        t = lambda y: y[..., 0].transpose(-1, -2)  # noqa: E731
        pool[p:p + c] = _pack(kc, ks[..., 0, :], kz[..., 0, :], vc.view(c, hkv, PAGE, d), t(vs), t(vz))
    tail = ((torch.randn(n, 2, hkv, PAGE, d, device="cuda", generator=g) + mu) * m).to(dt)
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    start = torch.tensor([0] + list(np.cumsum(blocks)), device="cuda")[:-1, None]
    col = torch.arange(width, device="cuda")
    table = torch.where(col < torch.tensor(blocks, device="cuda")[:, None], order[(start + col).clamp(max=pages - 1)],
                        torch.full((), -1, dtype=torch.int32, device="cuda"))
    return pool, tail, table.contiguous(), (m, mu)


def _rows(cached, new):
    """(sequence, position, slot in the table's row) of every new token, on the host."""
    seq = np.repeat(np.arange(len(new)), new)
    pos = np.concatenate([np.arange(c, c + m) for c, m in zip(cached, new)]) if len(new) else np.zeros(0, int)
    return seq.astype(np.int32), pos.astype(np.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    op = case["op"]
    if op == "norm_rope":
        n, hq, hkv, d, dt = case["tokens"], case["q_heads"], case["kv_heads"], case["d"], _dt(case)
        rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
        scale = 0.3 + 2 * torch.rand(n, 1, 1, device="cuda", generator=g)
        st = dict(case=case, q=(rnd(n, hq, d) * scale + 0.2).to(dt), k=(rnd(n, hkv, d) * scale).to(dt),
                  v=rnd(n, hkv, d).to(dt), qw=None, qb=None, kw=None, kb=None)
        if case["norm"] != "none":
            st.update(qw=(1 + 0.2 * rnd(d)).to(dt), kw=(1 + 0.2 * rnd(d)).to(dt))
        if case["norm"] == "layer":
            st.update(qb=(0.1 * rnd(d)).to(dt), kb=(0.1 * rnd(d)).to(dt))
        if case["rope"] == "2d":        # special tokens at (0, 0), patches by row and column
            at = (torch.arange(n, device="cuda") - 5).clamp(min=-1)
            yx = torch.stack([at // case["far"] + 1, at % case["far"] + 1], -1)
            st["positions"] = torch.where(at[:, None] < 0, torch.zeros_like(yx), yx).to(torch.int32).contiguous()
            st["inv_freq"] = 100.0 ** (-torch.arange(d // 4, device="cuda").float() / (d // 4))
        else:                           # a run of positions that ends at `far`
            first = max(0, case["far"] - n) if n > 1 else case["far"]
            st["positions"] = (first + torch.arange(n, device="cuda")).to(torch.int32)
            st["inv_freq"] = 500000.0 ** (-torch.arange(d // 2, device="cuda").float() / (d // 2))
        return st
    cached, new = _lengths(case)
    if op == "plan":
        most = [c + max(0, m) for c, m in zip(cached, new)]
        width = max(1, max(-(-h // PAGE) for h in most))
        have = [-(-c // PAGE) for c in cached]
        pages = sum(-(-h // PAGE) for h in most) + 17
        order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
        start = torch.tensor([0] + list(np.cumsum(have)), device="cuda")
        col = torch.arange(width, device="cuda")
        table = torch.where(col < torch.tensor(have, device="cuda")[:, None],
                            order[(start[:-1, None] + col).clamp(max=pages - 1)],
                            torch.full((), -1, dtype=torch.int32, device="cuda")).contiguous()
        used = sum(have)
        head = (5 + 3 * int(seed)) % pages         # the free pages lie in a ring, from its head on
        ring = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
        ring[(head + torch.arange(pages - used, device="cuda")) % pages] = order[used:]
        return dict(case=case, cached=_ints(cached), new=_ints(new), table=table, ring=ring,
                    state=_ints([head, pages - used, 0, 0]), max_tokens=sum(max(0, m) for m in new) + 9)
    held = [c + m for c, m in zip(cached, new)]
    pool, tail, table, (m, mu) = _cache(case, cached, held, g)
    hkv, d, dt = case["kv_heads"], case["d"], _dt(case)
    seq, pos = _rows(cached, new)
    st = dict(case=case, pages=pool, k_tail=tail, table=table, total=_ints(held), token_seq=torch.from_numpy(seq).cuda(),
              cu=_ints([0] + [int(x) for x in np.cumsum(new)]), positions=torch.from_numpy(pos).cuda())
    n = len(seq)
    if op == "append":
        st["k"] = ((torch.randn(n, hkv, d, device="cuda", generator=g) + mu.transpose(0, 1)) * m.transpose(0, 1)).to(dt)
        st["v"] = torch.randn(n, hkv, d, device="cuda", generator=g).to(dt)
        at = st["positions"].long()
        page = table[st["token_seq"].long(), at // PAGE].long()
        st["slots"] = (page * PAGE + at % PAGE).to(torch.int32)
        first = [c // PAGE * PAGE for c in cached]
        rseq, rpos = _rows(first, [h - f for h, f in zip(held, first)])
        st["read_seq"], st["read_pos"] = torch.from_numpy(rseq).cuda(), torch.from_numpy(rpos).cuda()
    else:
        st["q"] = torch.randn(n, case["q_heads"], d, device="cuda", generator=g).to(dt)
        st["max_new"] = max(new)
    return st


# ------------------------------------------------------------------------------------------------ plain forms
def _values(rec, d):
    """Keys and values (float32, [..., 64, d]) that records [..., 72 d] stand for."""
    lead = rec.shape[:-1]
    b = len(lead)
    at = lambda *o: tuple(range(b)) + tuple(b + i for i in o)  # noqa: E731
    nib = torch.stack([rec[..., :64 * d] & 15, rec[..., :64 * d] >> 4], -1)
    k = nib[..., :32 * d, :].reshape(*lead, d // 32, 2, 8, 4, 4, 2, 2, 2).permute(at(4, 7, 2, 0, 3, 1, 6, 5))
    v = nib[..., 32 * d:, :].reshape(*lead, 4, d // 64, 8, 4, 4, 2, 2, 2).permute(at(0, 6, 3, 5, 1, 2, 4, 7))
    par = rec[..., 64 * d:].contiguous().view(torch.float16).float().view(*lead, 4, d)
    k = k.reshape(*lead, PAGE, d).float() * par[..., 0, None, :] + par[..., 1, None, :]
    vs, vz = (par[..., i, :].view(*lead, d // 64, 8, 8).permute(at(2, 1, 0)).reshape(*lead, PAGE, d // 64, 1) for i in (2, 3))
    v = v.reshape(*lead, PAGE, d // 64, 64).float() * vs + vz
    return k, v.reshape(*lead, PAGE, d)


def _plain_norm_rope(st):
    c = st["case"]
    d, dt = c["d"], st["q"].dtype
    r = d // 2 if c["rope"] == "2d" else d                     # channels that one position rotates
    ang = st["positions"].double().view(c["tokens"], -1, 1) * st["inv_freq"].double()     # [n, 1 or 2, r / 2]
    cos, sin = ang.cos().float()[:, None], ang.sin().float()[:, None]

    def one(x, w, b):
        x = x.float()
        if c["norm"] == "layer":
            x = x - x.mean(-1, keepdim=True)
        if c["norm"] != "none":
            x = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w.float()
        if b is not None:
            x = x + b.float()
        y = x.view(*x.shape[:2], d // r, r)
        if c["rope"] == "pairs":
            lo, hi = y[..., 0::2], y[..., 1::2]
            y = torch.stack([lo * cos - hi * sin, hi * cos + lo * sin], -1)
        else:
            lo, hi = y[..., :r // 2], y[..., r // 2:]
            y = torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1)
        return lay(y.reshape(x.shape).to(dt))

    def lay(x):
        return x.transpose(0, 1).contiguous() if c["head_major"] else x.contiguous()

    return one(st["q"], st["qw"], st["qb"]), one(st["k"], st["kw"], st["kb"]), lay(st["v"].clone())


def _plain_plan(st):
    cached, new, table, ring = st["cached"].long().clamp(min=0), st["new"].long(), st["table"], st["ring"]
    head, count, pages, width, most = st["state"][0].long(), st["state"][1].long(), ring.numel(), table.shape[1], st["max_tokens"]
    gone, fresh = new < 0, new.clamp(min=0)
    cu = torch.cat([torch.zeros_like(fresh[:1]), fresh.cumsum(0)])
    have = (cached + PAGE - 1) // PAGE
    need = (cached + fresh + PAGE - 1) // PAGE - have
    bad = ~gone & ((have + need > width) | (fresh > 0) & (cu[1:] > most))
    need = torch.where(gone | bad, torch.zeros_like(need), need)
    before = need.cumsum(0) - need
    bad = bad | (need > 0) & (before + need > count)
    need = torch.where(bad, torch.zeros_like(need), need)
    freed = torch.where(gone, have.clamp(max=width), torch.zeros_like(have))
    fbefore = freed.cumsum(0) - freed
    total = torch.where(gone, torch.zeros_like(cached), torch.where(bad, cached, cached + fresh))
    cu = cu.clamp(max=most)
    t = torch.arange(most, device=cu.device)
    live = t < cu[-1]
    seq = torch.searchsorted(cu[1:].contiguous(), t, right=True).clamp(max=new.numel() - 1)
    pos = cached[seq] + t - cu[seq]
    block = pos // PAGE
    page = torch.where(block < have[seq], table[seq, block.clamp(max=width - 1)].long(),
                       ring[(head + before[seq] + block - have[seq]) % pages].long())
    slot = torch.where(live & ~bad[seq], page * PAGE + pos % PAGE, torch.full_like(pos, -1))
    col = torch.arange(width, device=cu.device)
    from_ring = ring[(head + before[:, None] + col - have[:, None]) % pages]
    table_out = torch.where((col >= have[:, None]) & (col < (have + need)[:, None]), from_ring, table)
    to = torch.where(col < freed[:, None], (head + count + fbefore[:, None] + col) % pages, torch.full_like(table, pages).long())
    ring_out = torch.cat([ring, ring[:1]]).scatter(0, to.view(-1), table.view(-1))[:pages]
    state = torch.stack([(head + need.sum()) % pages, count - need.sum() + freed.sum(), bad.sum(), cu[-1]])
    i32 = lambda x: x.to(torch.int32)  # noqa: E731
    return [table_out, ring_out, i32(state), i32(cu), i32(total), i32(slot),
            i32(torch.where(live, seq, torch.full_like(seq, -1))), i32(torch.where(live, pos, torch.zeros_like(pos)))]


def _plain_append(st):
    c, d, dt = st["case"], st["case"]["d"], st["k"].dtype
    seq, pos = st["read_seq"].long(), st["read_pos"].long()
    total, cu = st["total"].long(), st["cu"].long()
    cached = (total - (cu[1:] - cu[:-1]))[seq]
    old = (pos < cached)[:, None, None]
    row = (cu[seq] + pos - cached).clamp(min=0)
    k = torch.where(old, st["k_tail"][seq, pos // PAGE % 2, :, pos % PAGE].double(), st["k"][row].double())
    # values: those that were there come from the sequence's page, new ones are quantised per token
    first = (total - (cu[1:] - cu[:-1])) // PAGE
    held = st["table"].gather(1, first.clamp(max=st["table"].shape[1] - 1)[:, None])[:, 0].long().clamp(min=0)
    _, vold = _values(st["pages"][held], d)
    vc, vs, vz = _quantise(st["v"].double().view(-1, c["kv_heads"], d // 64, 64), -1)
    vnew = (vc * vs.double() + vz.double()).view(-1, c["kv_heads"], d)
    v = torch.where(old, vold[seq, :, pos % PAGE].double(), vnew[row])
    # keys: a filled page is quantised per channel over its 64 rows, an unfilled one stays
    page = (pos % PAGE == 0).long().cumsum(0) - 1
    groups = seq.numel() // PAGE + total.numel()
    x = k.clamp(-65504, 65504)
    lo = torch.full((groups, *x.shape[1:]), math.inf, dtype=x.dtype, device=x.device).index_reduce_(0, page, x, "amin")
    hi = torch.full_like(lo, -math.inf).index_reduce_(0, page, x, "amax")
    z = _down(lo)
    s = -_down(-((hi - z.double()) / 15))
    s = torch.where(s == 0, torch.ones_like(s), s).double()[page]
    z = z.double()[page]
    kq = ((x - z) / s).round().clamp(0, 15) * s + z
    k = torch.where((pos < total[seq] // PAGE * PAGE)[:, None, None], kq, k)
    return k.to(dt), v.to(dt)


def _plain_attention(st):
    c, dt = st["case"], st["q"].dtype
    hq, hkv, d = c["q_heads"], c["kv_heads"], c["d"]
    table, total, cu = st["table"], st["total"].long(), st["cu"].long()
    n, width, group, most = table.shape[0], table.shape[1], hq // hkv, st["max_new"]
    k, v = _values(st["pages"][table.clamp(min=0).long()], d)                 # [n, width, hkv, 64, d]
    last, all_ = total // PAGE, torch.arange(n, device=total.device)
    at = last.clamp(max=width - 1)
    raw = st["k_tail"][all_, last % 2].float()
    k[all_, at] = torch.where((last < width)[:, None, None, None], raw, k[all_, at])
    pos = torch.arange(width * PAGE, device=total.device)
    held = (pos < total[:, None])[:, None, :, None]
    k = torch.where(held, k.permute(0, 2, 1, 3, 4).reshape(n, hkv, -1, d), 0.0)
    v = torch.where(held, v.permute(0, 2, 1, 3, 4).reshape(n, hkv, -1, d), 0.0)
    i = torch.arange(most, device=total.device)
    row = (cu[:-1, None] + i).clamp(max=st["q"].shape[0] - 1)
    q = st["q"][row].float().view(n, most, hkv, group, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, most * group, d)
    s = q @ k.transpose(-1, -2) * (1 / math.sqrt(d))
    where = (total - (cu[1:] - cu[:-1]))[:, None] + i                          # position of each query
    seen = pos <= where[..., None]
    if c["window"]:
        seen = seen & (pos > where[..., None] - c["window"])
    s = s.view(n, hkv, most, group, -1).masked_fill(~seen[:, None, :, None], -math.inf)
    e = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-3e38))
    o = e.view(n, hkv, most * group, -1) @ v / e.sum(-1).view(n, hkv, -1, 1).clamp(min=1e-30)
    o = o.view(n, hkv, most, group, d).permute(0, 2, 1, 3, 4).reshape(n, most, hq, d)
    seq = st["token_seq"].long()
    return o[seq, torch.arange(seq.numel(), device=seq.device) - cu[seq]].to(dt)


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    op = st["case"]["op"]
    if own:
        from paper_2602_21780_b200 import binding
        if op == "norm_rope":
            c = st["case"]
            return binding.qk_norm_rope(st["q"], st["k"], st["v"], norm=c["norm"], q_weight=st["qw"], q_bias=st["qb"],
                                        k_weight=st["kw"], k_bias=st["kb"], eps=1e-6, rope=c["rope"],
                                        inv_freq=st["inv_freq"], positions=st["positions"], head_major=c["head_major"])
        if op == "plan":
            p = binding.page_plan(st["cached"], st["new"], st["table"], st["ring"], st["state"], st["max_tokens"])
            return [st["table"], st["ring"], p.ring_state, p.cu_new, p.total_len, p.slot_map, p.token_seq, p.positions]
        if op == "append":
            binding.page_append(st["pages"], st["k_tail"], st["k"], st["v"], st["slots"], st["token_seq"], st["cu"], st["total"])
            return binding.page_read(st["pages"], st["k_tail"], st["table"], st["total"], st["read_seq"], st["read_pos"])
        return binding.page_attention(st["q"], st["pages"], st["k_tail"], st["table"], st["cu"], st["total"],
                                      st["max_new"], window=st["case"]["window"])
    return {"norm_rope": _plain_norm_rope, "plan": _plain_plan, "append": _plain_append,
            "attention": _plain_attention}[op](st)


# ------------------------------------------------------------------------------------------------ 64 bits
def _exact_record(rec, d):
    """Keys and values (float64, [..., 64, d]) of records, token by token and channel by channel from the byte that
    holds each."""
    dev = rec.device
    t, ch = torch.arange(PAGE, device=dev)[:, None], torch.arange(d, device=dev)[None, :]
    kb = (ch // 32 * 2 + ch % 8 // 4) * 512 + (t % 8) * 64 + (ch % 32 // 8) * 16 + (t // 16) * 4 + (ch % 2) * 2 + ch % 4 // 2
    vb = 32 * d + (t // 16) * 8 * d + (ch // 64) * 512 + (ch % 64 // 8) * 64 + (t % 8 // 2) * 16 + (ch % 8 // 2) * 4 + (t % 2) * 2 + t % 16 // 8
    kn, vn = (t // 8 % 2 * 4).expand(PAGE, d), (ch % 2 * 4).expand(PAGE, d)
    codes = [((rec[..., b.reshape(-1)].to(torch.int32) >> s.reshape(-1)) & 15).double().view(*rec.shape[:-1], PAGE, d)
             for b, s in ((kb, kn), (vb, vn))]
    f = rec[..., 64 * d:].contiguous().view(torch.float16).double()
    at = (ch // 64 * PAGE + t % 8 * 8 + t // 8).reshape(-1)
    pick = lambda o: f[..., o + at].view(*rec.shape[:-1], PAGE, d)  # noqa: E731
    return (codes[0] * f[..., None, :d] + f[..., None, d:2 * d], codes[1] * pick(2 * d) + pick(3 * d))


def _exact_down(x):
    """The largest float16 not above each x, looked up among all of them."""
    bits = torch.arange(-32768, 32768, device=x.device).to(torch.int16)
    every = bits.view(torch.float16).double()
    every = every[every.isfinite()].sort().values
    return every[torch.searchsorted(every, x.contiguous(), right=True) - 1]


def _exact_group(x, dim):
    lo, hi = x.min(dim, keepdim=True).values, x.max(dim, keepdim=True).values
    z = _exact_down(lo)
    s = -_exact_down((z - hi) / 15)
    s[s == 0] = 1
    return torch.clamp(torch.round((x - z) / s), 0, 15) * s + z


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "norm_rope":
        n, d = case["tokens"], case["d"]
        p = st["positions"].double().view(n, -1)

        def turn(x, at):                      # x [n, h, 2, r / 2] -> rotated as complex numbers
            a = at[:, None] * st["inv_freq"].double()
            y = torch.complex(x[:, :, 0], x[:, :, 1]) * torch.polar(torch.ones_like(a), a)[:, None]
            return torch.stack([y.real, y.imag], 2)

        def one(x, w, b):
            x = x.double()
            if case["norm"] == "layer":
                x = (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + 1e-6)
            elif case["norm"] == "rms":
                x = x * torch.rsqrt((x * x).sum(-1, keepdim=True) / d + 1e-6)
            x = x * w.double() if w is not None else x
            x = x + b.double() if b is not None else x
            h = x.shape[1]
            if case["rope"] == "pairs":
                x = turn(x.view(n, h, d // 2, 2).transpose(2, 3), p[:, 0]).transpose(2, 3).reshape(n, h, d)
            elif case["rope"] == "half":
                x = turn(x.view(n, h, 2, d // 2), p[:, 0]).reshape(n, h, d)
            else:
                x = torch.cat([turn(x[..., i * d // 2:(i + 1) * d // 2].reshape(n, h, 2, d // 4), p[:, i]).reshape(n, h, -1)
                               for i in (0, 1)], -1)
            return x.permute(1, 0, 2) if case["head_major"] else x

        v = st["v"].double()
        return one(st["q"], st["qw"], st["qb"]), one(st["k"], st["kw"], st["kb"]), v.permute(1, 0, 2) if case["head_major"] else v
    if case["op"] == "plan":                  # step by step on the host
        cached, new, table, ring, state = (st[k].cpu().numpy().copy() for k in ("cached", "new", "table", "ring", "state"))
        pages, most = len(ring), st["max_tokens"]
        head, left, free = int(state[0]), int(state[1]), int(state[0]) + int(state[1])
        cu, total, slot, seq, pos, refused = [0], [], [], [], [], 0
        for s, (c, m) in enumerate(zip(cached.tolist(), new.tolist())):
            have = -(-c // PAGE)
            if m < 0:
                for b in range(have):
                    ring[free % pages] = table[s, b]
                    free += 1
                m, grown = 0, 0
            else:
                need = -(-(c + m) // PAGE) - have
                ok = have + need <= table.shape[1] and need <= left
                for b in range(need if ok else 0):
                    table[s, have + b] = ring[head % pages]
                    head, left = head + 1, left - 1
                refused += not ok
                grown = c + m if ok else c
                for i in range(c, c + m):
                    slot.append(int(table[s, i // PAGE]) * PAGE + i % PAGE if ok else -1)
                    seq.append(s)
                    pos.append(i)
            cu.append(cu[-1] + m)
            total.append(grown)
        pad = most - len(slot)
        out = [table, ring, [head % pages, free - head, refused, len(slot)], cu, total, slot + [-1] * pad, seq + [-1] * pad, pos + [0] * pad]
        return [np.asarray(x, dtype=np.int32) for x in out]
    hkv, d = case["kv_heads"], case["d"]
    cached, new = _lengths(case)
    cu = [0] + [int(x) for x in np.cumsum(new)]
    if case["op"] == "append":
        ks, vs = [], []
        for s, (c, m) in enumerate(zip(cached, new)):
            first, end = c // PAGE, c + m
            rec = st["pages"][st["table"][s, first].long()] if c % PAGE else None
            k = torch.cat([st["k_tail"][s, first % 2, :, :c % PAGE].transpose(0, 1), st["k"][cu[s]:cu[s + 1]]]).double()
            full = (end - first * PAGE) // PAGE * PAGE
            k[:full] = _exact_group(k[:full].view(-1, PAGE, hkv, d), 1).view(full, hkv, d) if full else k[:full]
            v = _exact_group(st["v"][cu[s]:cu[s + 1]].double().view(-1, hkv, d // 64, 64), -1).view(-1, hkv, d)
            if rec is not None:
                v = torch.cat([_exact_record(rec, d)[1][:, :c % PAGE].transpose(0, 1), v])
            ks.append(k)
            vs.append(v)
        return torch.cat(ks), torch.cat(vs)
    outs, group = [], case["q_heads"] // hkv
    for s, (c, m) in enumerate(zip(cached, new)):
        end = c + m
        k, v = _exact_record(st["pages"][st["table"][s, :-(-end // PAGE)].long()], d)      # [pages, hkv, 64, d]
        if end % PAGE:
            k[-1] = st["k_tail"][s, end // PAGE % 2].double()
        k, v = (x.transpose(0, 1).reshape(hkv, -1, d)[:, :end] for x in (k, v))
        q = st["q"][cu[s]:cu[s + 1]].double().view(m, hkv, group, d)
        out = torch.empty_like(q)
        key = torch.arange(end, device=q.device)
        for a in range(0, m, 256):
            b = min(m, a + 256)
            at = c + torch.arange(a, b, device=q.device)[:, None]
            seen = (key <= at) & (key > at - case["window"] if case["window"] else key >= 0)
            w = torch.einsum("nhgd,htd->hgnt", q[a:b], k) / math.sqrt(d)
            w = torch.softmax(w.masked_fill(~seen, -math.inf), -1)
            out[a:b] = torch.einsum("hgnt,htd->nhgd", w, v)
        outs.append(out.view(m, case["q_heads"], d))
    return torch.cat(outs)
