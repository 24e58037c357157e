"""Operators over a pool of 8-bit pages, and rotary positions with several axes: what each is asked to do, its plain form
in elementary torch operations, and the sizes it is used at.

  axes        queries and keys normalised per head and rotated by several positions a token (time, height, width)
  append8     new keys and values quantised into 8-bit pages of 64 tokens, and the touched pages read back as values
  attention8  ragged causal attention (grouped heads, one or many new tokens per sequence) over the pages
  select      the pages that each new token attends to, by a score of the token's queries against the pages' mean keys
  selected    attention of each new token over its selected pages

A page record holds 64 tokens of one key/value head, 130 * head_dim bytes:
  [0, 64 d)                 e4m3 key codes in 16-byte pieces [8 a][d/64 c][8 g][4 j]: token 8 a + g, channels 64 c + 16 j and
                            the 15 after it
  [64 d, 64 d + 12)         float32: key scale, value scale, factor of the mean key
  [64 d + 32, 128 d + 32)   e4m3 value codes in pieces of d/8 bytes [4 t][2 b][2 h][8 g][4 j]: token 16 t + 8 b + 2 j + h,
                            channels (d/8) g and the d/8 - 1 after it
  [128 d + 32, 129 d + 32)  int8 mean key [d] of a full page
A value is code * scale.  A scale is 2^e with the smallest e in [-80, 8] for which 448 * 2^e reaches the largest magnitude
(inputs beyond 65504 count as 65504) that the page has been given, code = nearest-even e4m3 of x / 2^e; codes of an unfilled
page are rescaled when later tokens raise e.  Mean key: S = sum of a channel's 64 codes, A = max |S|, int8 code =
nearest-even of S * (127 / A) in float32, factor = A * scale / 64.
Score of a page for a token and key/value head: the largest over the group's query heads of (dot * factor) * a, with
a = max(max |q|, 2^-60), q8 = nearest-even of q * (127 / a), dot = sum of q8 * mean codes, each product float32.
"""
import math

import numpy as np
import torch

own = False

PAGE = 64


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one decoded token with a text position on all three axes: latency is all there is
        dict(name="axes one token", op="axes", tokens=1, q_heads=32, kv_heads=8, d=128, norm="rms", rope="half", mixed=False,
             dtype="bf16"),
        # six video frames of 37 x 37 patches behind a prompt, rotated by time, row and column
        dict(name="axes video 8219", op="axes", tokens=8219, q_heads=32, kv_heads=8, d=128, norm="rms", rope="half", mixed=True,
             dtype="bf16"),
        # decode step of a batch
        dict(name="append8 decode 256", op="append8", seqs=256, cached_lo=65, cached_hi=4000, new_lo=1, new_hi=1, kv_heads=8,
             d=128, dtype="bf16"),
        # prompts of ragged lengths, continued from page boundaries
        dict(name="append8 prompts 5", op="append8", seqs=5, cached_lo=0, cached_hi=2048, new_lo=1500, new_hi=9001, kv_heads=8,
             d=64, dtype="fp16"),
        # one short sequence, one token: latency
        dict(name="attention8 one of 261", op="attention8", seqs=1, total_lo=261, total_hi=261, new_lo=1, new_hi=1, q_heads=16,
             kv_heads=16, d=64, window=0, dtype="fp16"),
        # a decode batch of ragged lengths, grouped heads
        dict(name="attention8 decode 64", op="attention8", seqs=64, total_lo=900, total_hi=16000, new_lo=1, new_hi=1, q_heads=32,
             kv_heads=8, d=128, window=0, dtype="bf16"),
        # one very long sequence, four tokens at once (drafted tokens being verified)
        dict(name="attention8 4 of 200001", op="attention8", seqs=1, total_lo=200001, total_hi=200001, new_lo=4, new_hi=4,
             q_heads=32, kv_heads=8, d=128, window=0, dtype="bf16"),
        # ragged chunks of prompts, grouped heads
        dict(name="attention8 chunks 6", op="attention8", seqs=6, total_lo=2100, total_hi=9000, new_lo=300, new_hi=2047,
             q_heads=32, kv_heads=8, d=128, window=0, dtype="bf16"),
        # the selection of a decode batch of long ragged sequences
        dict(name="select decode 16", op="select", seqs=16, total_lo=2000, total_hi=60000, new_lo=1, new_hi=1, q_heads=32,
             kv_heads=8, d=128, top=32, first=1, recent=2, dtype="bf16"),
        # a chunk of a prompt behind a long context, every token with a selection of its own
        dict(name="select chunk 1021", op="select", seqs=1, total_lo=40000, total_hi=40000, new_lo=1021, new_hi=1021, q_heads=32,
             kv_heads=8, d=128, top=32, first=1, recent=2, dtype="bf16"),
        # a decode batch of long sequences over 2048 tokens each
        dict(name="selected decode 32", op="selected", seqs=32, total_lo=4000, total_hi=30000, new_lo=1, new_hi=1, q_heads=32,
             kv_heads=8, d=128, top=32, first=1, recent=2, dtype="bf16"),
        # a chunk of a prompt over the pages that each of its tokens selected
        dict(name="selected chunk 509", op="selected", seqs=1, total_lo=25000, total_hi=25000, new_lo=509, new_hi=509, q_heads=32,
             kv_heads=8, d=128, top=24, first=1, recent=2, dtype="fp16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["axes", "append8", "attention8", "attention8", "select", "selected"])
    dtype = rng.choice(["bf16", "fp16"])
    q_heads, kv_heads, d = rng.choice([(32, 8, 128), (16, 16, 64), (8, 1, 128), (20, 4, 128), (12, 4, 64), (5, 5, 64)])
    heads = dict(q_heads=q_heads, kv_heads=kv_heads, d=d)
    if op == "axes":
        return dict(op=op, tokens=_log(rng, 1, 8000), **heads, norm=rng.choice(["rms", "layer", "none"]),
                    rope=rng.choice(["half", "pairs"]), mixed=rng.random() < 0.5, dtype=dtype)
    if op == "append8":
        if rng.random() < 0.5:
            return dict(op=op, seqs=_log(rng, 1, 256), cached_lo=0, cached_hi=_log(rng, 50, 3000), new_lo=1,
                        new_hi=rng.choice([1, 1, 2, 5]), kv_heads=kv_heads, d=d, dtype=dtype)
        return dict(op=op, seqs=rng.randint(1, 6), cached_lo=0, cached_hi=_log(rng, 64, 2000), new_lo=70,
                    new_hi=_log(rng, 100, 6000), kv_heads=kv_heads, d=d, dtype=dtype)
    if op == "attention8":
        window = 0 if rng.random() < 0.7 else _log(rng, 100, 5000)
        if rng.random() < 0.6:
            seqs = _log(rng, 1, 64)
            hi = _log(rng, 60, 15000 if seqs > 8 else 90000 // seqs)
            return dict(op=op, seqs=seqs, total_lo=max(8, hi // rng.choice([1, 3, 10])), total_hi=hi, new_lo=1,
                        new_hi=rng.choice([1, 1, 1, 2, 7]), **heads, window=window, dtype=dtype)
        seqs, new_hi = rng.randint(1, 5), _log(rng, 40, 1300)
        return dict(op=op, seqs=seqs, total_lo=new_hi, total_hi=new_hi + _log(rng, 10, 6000), new_lo=max(1, new_hi // 4),
                    new_hi=new_hi, **heads, window=window, dtype=dtype)
    first, recent = rng.choice([0, 1, 2]), rng.choice([1, 2, 4])
    top = max(first + recent, _log(rng, 4, 32))
    if rng.random() < 0.6:
        seqs = _log(rng, 1, 32)
        hi = _log(rng, 200, 24000 if seqs > 8 else 120000 // seqs)
        return dict(op=op, seqs=seqs, total_lo=max(8, hi // rng.choice([1, 3, 10])), total_hi=hi, new_lo=1,
                    new_hi=rng.choice([1, 1, 1, 2, 5]), **heads, top=top, first=first, recent=recent, dtype=dtype)
    seqs, new_hi = rng.randint(1, 3), _log(rng, 20, 160)
    return dict(op=op, seqs=seqs, total_lo=new_hi, total_hi=new_hi + _log(rng, 200, 24000), new_lo=max(1, new_hi // 3),
                new_hi=new_hi, **heads, top=top, first=first, recent=recent, dtype=dtype)


# A case's ragged lengths are a function of the case alone, spread over [lo, hi]; a single sequence has the upper end.
def _spread(i, n, lo, hi):
    if n == 1 or hi <= lo:
        return hi
    return lo + (((i * 2654435761 + 40503) % 4294967296) * (hi - lo + 1) >> 32)


def _lengths(case):
    """Per sequence: (tokens cached before the call, new tokens)."""
    n = case["seqs"]
    new = [_spread(3 * i + 1, n, case["new_lo"], case["new_hi"]) for i in range(n)]
    if case["op"] != "append8":
        total = [_spread(i, n, case["total_lo"], case["total_hi"]) for i in range(n)]
        return [max(0, t - m) for t, m in zip(total, new)], new
    cached = [_spread(i, n, case["cached_lo"], case["cached_hi"]) for i in range(n)]
    # chunks of a prompt end at a page's end; a few decoded tokens start anywhere
    return [c // PAGE * PAGE if m > PAGE else c for c, m in zip(cached, new)], new


def work(case):
    op, d = case["op"], case["d"]
    if op == "axes":
        rows = case["tokens"] * (case["q_heads"] + 2 * case["kv_heads"])
        return dict(bytes=4 * rows * d + 12 * case["tokens"], flops=10 * rows * d)
    cached, new = _lengths(case)
    hkv, n = case["kv_heads"], sum(new)
    if op == "append8":
        back = sum(c + m - c // PAGE * PAGE for c, m in zip(cached, new))
        # new rows read, codes written, the touched pages read back and written out as values
        return dict(bytes=hkv * d * (4 * n + 2 * n + 2 * back + 4 * back), flops=hkv * d * (6 * n + 2 * back))
    hq = case["q_heads"]
    if op == "attention8":
        w, held, pairs = case["window"], 0, 0
        for c, m in zip(cached, new):
            held += c + m - (max(0, c - w + 1) if w else 0)
            pairs += sum(min(c + i + 1, w) if w else c + i + 1 for i in range(m))
        return dict(bytes=2 * hkv * d * held + 4 * n * hq * d, flops=4 * pairs * hq * d)
    pages = [[(c + i) // PAGE + 1 for i in range(m)] for c, m in zip(cached, new)]
    if op == "select":
        # mean keys once a sequence and head, queries, the list
        seen = sum(max(p, default=0) for p in pages)
        return dict(bytes=hkv * seen * (d + 4) + 2 * n * hq * d + 4 * n * hkv * case["top"],
                    flops=2 * sum(map(sum, pages)) * hq * d)
    # a page that several tokens of a head select need not be read more than once
    many = sum(min(p[-1], case["top"] * len(p)) for p in pages if p)
    return dict(bytes=2 * hkv * d * PAGE * many + 4 * n * hq * d + 4 * n * hkv * case["top"],
                flops=4 * PAGE * sum(min(x, case["top"]) for p in pages for x in p) * hq * d)


# ------------------------------------------------------------------------------------------------ inputs
def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _scale(amax):
    """The power of two for a page's largest magnitude (float32)."""
    m, e = torch.frexp(amax.float().clamp(max=65504))         # m in [0.5, 1)
    e = e - 9 + (m > 0.875)
    e = torch.where(amax > 0, e, torch.full_like(e, -80)).clamp(-80, 8)
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _over(a):
    """127 / a, rounded once, and 0 where a is."""
    return torch.where(a > 0, torch.div(torch.full_like(a, 127), a), torch.zeros_like(a))


def _e4m3(y):
    """The nearest e4m3 value of y (float32), as float32."""
    return y.clamp(-448, 448).to(torch.float8_e4m3fn).float()


def _pack(k, v, ks, vs):
    """Records [..., 130 d] of codes (float32 values of e4m3) [..., 64, d] and scales [...]."""
    lead, d = k.shape[:-2], k.shape[-1]
    b = len(lead)
    at = lambda *o: tuple(range(b)) + tuple(b + i for i in o)  # noqa: E731
    kb = k.to(torch.float8_e4m3fn).view(torch.uint8).view(*lead, 8, 8, d // 64, 4, 16).permute(at(0, 2, 1, 3, 4))
    vb = v.to(torch.float8_e4m3fn).view(torch.uint8).view(*lead, 4, 2, 4, 2, 8, d // 8).permute(at(0, 1, 3, 4, 2, 5))
    total = k.sum(-2)                                          # exact: whole numbers of 2^-9 below 2^15
    top = total.abs().amax(-1)
    mean = (total * _over(top)[..., None]).round().to(torch.int8)
    rec = torch.zeros(*lead, 130 * d, dtype=torch.uint8, device=k.device)
    rec[..., :64 * d] = kb.reshape(*lead, 64 * d)
    rec[..., 64 * d:64 * d + 12] = torch.stack([ks, vs, top * ks / 64], -1).float().view(torch.uint8)
    rec[..., 64 * d + 32:128 * d + 32] = vb.reshape(*lead, 64 * d)
    rec[..., 128 * d + 32:129 * d + 32] = mean.view(torch.uint8)
    return rec


def _cache(case, held, g):
    """Pool and block table of sequences that hold `held` tokens."""
    hkv, d, dt, n = case["kv_heads"], case["d"], _dt(case), case["seqs"]
    blocks = [-(-h // PAGE) for h in held]
    width, pages = max(1, max(blocks)), sum(blocks) + 3
    # keys after their norm: per-channel weights, a few channels large, offsets of their own; values plain
    m = 0.6 + 0.8 * torch.rand(hkv, 1, d, device="cuda", generator=g)
    m[:, :, torch.randint(0, d, (3,), device="cuda", generator=g)] *= 3
    mu = 0.5 * torch.randn(hkv, 1, d, device="cuda", generator=g)
    pool = torch.empty(pages, hkv, 130 * d, dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // (hkv * PAGE * d))
    for p in range(0, pages, step):
        c = min(step, pages - p)
        # neighbouring tokens resemble each other: a page has a direction of its own
        own_k = 0.4 * torch.randn(c, hkv, 1, d, device="cuda", generator=g)
        k = ((torch.randn(c, hkv, PAGE, d, device="cuda", generator=g) + own_k + mu) * m).to(dt).float()
        v = torch.randn(c, hkv, PAGE, d, device="cuda", generator=g).to(dt).float()
        ks, vs = _scale(k.abs().amax((-1, -2))), _scale(v.abs().amax((-1, -2)))
        pool[p:p + c] = _pack(_e4m3(k / ks[..., None, None]), _e4m3(v / vs[..., None, None]), ks, vs)
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    start = torch.tensor([0] + list(np.cumsum(blocks)), device="cuda")[:-1, None]
    col = torch.arange(width, device="cuda")
    table = torch.where(col < torch.tensor(blocks, device="cuda")[:, None], order[(start + col).clamp(max=pages - 1)],
                        torch.full((), -1, dtype=torch.int32, device="cuda"))
    return pool, table.contiguous(), (m, mu)


def _rows(cached, new):
    """(sequence, position) of every new token, on the host."""
    seq = np.repeat(np.arange(len(new)), new)
    pos = np.concatenate([np.arange(c, c + m) for c, m in zip(cached, new)]) if len(new) else np.zeros(0, int)
    return seq.astype(np.int32), pos.astype(np.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    op, dt, d, hkv = case["op"], _dt(case), case["d"], case["kv_heads"]
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    if op == "axes":
        n, hq = case["tokens"], case["q_heads"]
        scale = 0.3 + 2 * torch.rand(n, 1, 1, device="cuda", generator=g)
        st = dict(case=case, q=(rnd(n, hq, d) * scale + 0.2).to(dt), k=(rnd(n, hkv, d) * scale).to(dt), v=rnd(n, hkv, d).to(dt),
                  qw=None, qb=None, kw=None, kb=None)
        if case["norm"] != "none":
            st.update(qw=(1 + 0.2 * rnd(d)).to(dt), kw=(1 + 0.2 * rnd(d)).to(dt))
        if case["norm"] == "layer":
            st.update(qb=(0.1 * rnd(d)).to(dt), kb=(0.1 * rnd(d)).to(dt))
        # a prompt's tokens have one position on all axes, then frames of 37 x 37 patches by time, row and column
        first = 20000 + 7 * (int(seed) % 11)
        i = torch.arange(n, device="cuda")
        p = (i - 5).clamp(min=0)
        at = torch.stack([p // 1369, p // 37 % 37, p % 37], -1) + first + 5
        st["positions"] = torch.where(i[:, None] < 5, (first + i)[:, None], at).to(torch.int32).contiguous()
        # frequencies of the axes: in a row (an eighth, then three eighths each, of the half head), or in turn
        f = torch.arange(d // 2, device="cuda")
        st["axes"] = ((f % 3) if case["mixed"] else (f >= d // 8).long() + (f >= 5 * d // 16).long()).to(torch.int32)
        st["inv_freq"] = 500000.0 ** (-f.float() / (d // 2))
        return st
    cached, new = _lengths(case)
    held = [c + m for c, m in zip(cached, new)]
    pool, table, (m, mu) = _cache(case, held, g)
    seq, pos = _rows(cached, new)
    n = len(seq)
    st = dict(case=case, pages=pool, table=table, total=_ints(held), token_seq=torch.from_numpy(seq).cuda(),
              cu=_ints([0] + [int(x) for x in np.cumsum(new)]), positions=torch.from_numpy(pos).cuda())
    if op == "append8":
        st["k"] = ((rnd(n, hkv, d) + mu.transpose(0, 1)) * m.transpose(0, 1)).to(dt)
        st["v"] = rnd(n, hkv, d).to(dt)
        at = st["positions"].long()
        page = table[st["token_seq"].long(), at // PAGE].long()
        st["slots"] = (page * PAGE + at % PAGE).to(torch.int32)
        first = [c // PAGE * PAGE for c in cached]
        rseq, rpos = _rows(first, [h - f for h, f in zip(held, first)])
        st["read_seq"], st["read_pos"] = torch.from_numpy(rseq).cuda(), torch.from_numpy(rpos).cuda()
        return st
    st["q"] = rnd(n, case["q_heads"], d).to(dt)
    st["max_new"] = max(new)
    if op == "selected":
        st["selected"] = _plain_select(st)
    return st


# ------------------------------------------------------------------------------------------------ plain forms
def _values(rec, d):
    """Keys and values (float32, [..., 64, d]) that records [..., 130 d] stand for."""
    lead = rec.shape[:-1]
    b = len(lead)
    at = lambda *o: tuple(range(b)) + tuple(b + i for i in o)  # noqa: E731
    f8 = lambda x: x.contiguous().view(torch.float8_e4m3fn).float()  # noqa: E731
    k = f8(rec[..., :64 * d]).view(*lead, 8, d // 64, 8, 4, 16).permute(at(0, 2, 1, 3, 4)).reshape(*lead, PAGE, d)
    v = f8(rec[..., 64 * d + 32:128 * d + 32]).view(*lead, 4, 2, 2, 8, 4, d // 8).permute(at(0, 1, 4, 2, 3, 5)).reshape(*lead, PAGE, d)
    s = rec[..., 64 * d:64 * d + 8].contiguous().view(torch.float32)
    return k * s[..., :1, None], v * s[..., 1:, None]


def _plain_axes(st):
    c = st["case"]
    d, dt = c["d"], st["q"].dtype
    ang = st["positions"][:, st["axes"].long()].double() * st["inv_freq"].double()          # [n, d / 2]
    cos, sin = ang.cos().float()[:, None], ang.sin().float()[:, None]

    def one(x, w, b):
        x = x.float()
        if c["norm"] == "layer":
            x = x - x.mean(-1, keepdim=True)
        if c["norm"] != "none":
            x = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w.float()
        if b is not None:
            x = x + b.float()
        if c["rope"] == "pairs":
            lo, hi = x[..., 0::2], x[..., 1::2]
            return torch.stack([lo * cos - hi * sin, hi * cos + lo * sin], -1).reshape(x.shape).to(dt)
        lo, hi = x[..., :d // 2], x[..., d // 2:]
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1).to(dt)

    return one(st["q"], st["qw"], st["qb"]), one(st["k"], st["kw"], st["kb"]), st["v"].clone()


def _plain_append(st):
    d, dt, table = st["case"]["d"], st["k"].dtype, st["table"]
    seq, pos = st["read_seq"].long(), st["read_pos"].long()
    total, cu = st["total"].long(), st["cu"].long()
    cached = total - (cu[1:] - cu[:-1])
    old = pos < cached[seq]
    begun = pos // PAGE * PAGE < cached[seq]                   # pages that held tokens before the call
    row = (cu[seq] + pos - cached[seq]).clamp(min=0)
    rec = st["pages"][table.gather(1, (cached // PAGE).clamp(max=table.shape[1] - 1)[:, None])[:, 0].long().clamp(min=0)]
    page = (pos % PAGE == 0).long().cumsum(0) - 1
    most = 65504 if dt == torch.float16 else 1e6

    def one(x, before, was):
        new = x[row].float().clamp(-65504, 65504)
        mag = torch.where(old[:, None], torch.zeros_like(new[..., 0]), new.abs().amax(-1))
        top = torch.zeros(seq.numel() // PAGE + total.numel(), mag.shape[1], device=mag.device).index_reduce_(0, page, mag, "amax")
        s = torch.maximum(_scale(top)[page], torch.where(begun[:, None], was[seq], torch.zeros_like(was[seq])))[..., None]
        y = torch.where(old[:, None, None], before[seq, :, pos % PAGE], new)
        return (_e4m3(y / s) * s).clamp(-most, most).to(dt)

    scales = rec[..., 64 * d:64 * d + 8].contiguous().view(torch.float32)
    k, v = _values(rec, d)
    return one(st["k"], k, scales[..., 0]), one(st["v"], v, scales[..., 1])


def _plain_attention(st):
    c, dt = st["case"], st["q"].dtype
    hq, hkv, d = c["q_heads"], c["kv_heads"], c["d"]
    table, total, cu = st["table"], st["total"].long(), st["cu"].long()
    n, width, group, most = table.shape[0], table.shape[1], hq // hkv, st["max_new"]
    k, v = _values(st["pages"][table.clamp(min=0).long()], d)                 # [n, width, hkv, 64, d]
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


def _plain_select(st):
    c = st["case"]
    hkv, d, top, first, recent = c["kv_heads"], c["d"], c["top"], c["first"], c["recent"]
    q, table, seq, mine = st["q"].float(), st["table"], st["token_seq"].long(), st["positions"].long() // PAGE
    n, width = q.shape[0], table.shape[1]
    a = q.abs().amax(-1).clamp(min=2.0 ** -60)
    q8 = (q * _over(a)[..., None]).round().view(n, hkv, -1, d)
    heads = st["pages"][table.clamp(min=0).long()][..., 64 * d + 8:64 * d + 12]                    # [seqs, width, hkv, 4]
    factor = heads.contiguous().view(torch.float32)[..., 0].permute(0, 2, 1)                       # [seqs, hkv, width]
    mean = st["pages"][..., 128 * d + 32:129 * d + 32][table.clamp(min=0).long()].contiguous().view(torch.int8).float().permute(0, 2, 3, 1)
    one = table.shape[0] == 1
    dot = (q8.transpose(0, 1) @ mean[0][:, None] if one else q8.transpose(0, 1) @ mean[seq].transpose(0, 1)).transpose(0, 1)    # whole numbers below 2^24
    score = (dot * factor[seq][:, :, None] * a.view(n, hkv, -1, 1)).amax(2)                        # [n, hkv, width]
    page = torch.arange(width, device=q.device)
    forced = (page < first) | (page > mine[:, None] - recent)
    seen = page <= mine[:, None]
    score = torch.where((forced & seen)[:, None], math.inf, score.masked_fill(~seen[:, None], -math.inf))
    best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :top]
    best = torch.where(best <= mine[:, None, None], best, torch.full_like(best, width))
    best = torch.cat([best, best.new_full((n, hkv, max(0, top - width)), width)], -1).sort(-1).values
    return torch.where(best < width, best, torch.full_like(best, -1)).to(torch.int32)


def _plain_selected(st):
    c, dt = st["case"], st["q"].dtype
    hkv, d, n, sel = c["kv_heads"], c["d"], st["q"].shape[0], st["selected"].long()
    page = st["table"][st["token_seq"].long()[:, None, None], sel.clamp(min=0)].long()             # [n, hkv, top]
    rec = st["pages"][page, torch.arange(hkv, device=sel.device)[:, None]]                         # [n, hkv, top, 130 d]
    k, v = (x.reshape(n, hkv, -1, d) for x in _values(rec, d))
    at = sel[..., None] * PAGE + torch.arange(PAGE, device=sel.device)
    seen = ((sel >= 0)[..., None] & (at <= st["positions"].long()[:, None, None, None])).reshape(n, hkv, 1, -1)
    k, v = (torch.where(seen[:, :, 0, :, None], x, 0.0) for x in (k, v))
    s = st["q"].float().view(n, hkv, -1, d) @ k.transpose(-1, -2) * (1 / math.sqrt(d))
    s = s.masked_fill(~seen, -math.inf)
    e = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-3e38))
    return (e @ v / e.sum(-1, keepdim=True).clamp(min=1e-30)).reshape(n, -1, d).to(dt)


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    op = st["case"]["op"]
    if own:
        from paper_2602_21780_b200 import binding
        c = st["case"]
        if op == "axes":
            return binding.qk_norm_rope(st["q"], st["k"], st["v"], norm=c["norm"], q_weight=st["qw"], q_bias=st["qb"],
                                        k_weight=st["kw"], k_bias=st["kb"], eps=1e-6, rope=c["rope"], inv_freq=st["inv_freq"],
                                        positions=st["positions"], axes=st["axes"])
        if op == "append8":
            binding.page8_append(st["pages"], st["k"], st["v"], st["slots"], st["token_seq"], st["cu"], st["total"])
            return binding.page8_read(st["pages"], st["table"], st["total"], st["read_seq"], st["read_pos"], st["k"].dtype)
        if op == "attention8":
            return binding.page8_attention(st["q"], st["pages"], st["table"], st["cu"], st["total"], st["max_new"],
                                           window=c["window"])
        if op == "select":
            return binding.page8_select(st["q"], st["pages"], st["table"], st["token_seq"], st["positions"], c["top"],
                                        first=c["first"], recent=c["recent"])
        return binding.page8_attention_selected(st["q"], st["pages"], st["table"], st["token_seq"], st["positions"],
                                                st["selected"])
    return {"axes": _plain_axes, "append8": _plain_append, "attention8": _plain_attention, "select": _plain_select,
            "selected": _plain_selected}[op](st)


# ------------------------------------------------------------------------------------------------ 64 bits
def _exact_e4m3():
    """Every finite e4m3 value by its code (NaN elsewhere), float64."""
    code = torch.arange(256, device="cuda")
    e, m = code >> 3 & 15, (code & 7).double()
    mag = torch.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * torch.exp2(e.double() - 7))
    mag[(code & 127) == 127] = math.nan
    return torch.where(code > 127, -mag, mag)


def _exact_record(rec, d):
    """Keys and values (float64, [..., 64, d]) of records, token by token and channel by channel from the byte that
    holds each."""
    dev = rec.device
    t, ch = torch.arange(PAGE, device=dev)[:, None], torch.arange(d, device=dev)[None, :]
    kb = t // 8 * 8 * d + ch // 64 * 512 + t % 8 * 64 + ch % 64
    w = d // 8
    vb = 64 * d + 32 + (t // 16 * 128 + t // 8 % 2 * 64 + t % 2 * 32 + ch // w * 4 + t % 8 // 2) * w + ch % w
    s = rec[..., 64 * d:64 * d + 8].contiguous().view(torch.float32).double()
    of = _exact_e4m3()
    return [of[rec[..., b.reshape(-1)].long()].view(*rec.shape[:-1], PAGE, d) * s[..., i, None, None] for i, b in enumerate((kb, vb))]


def _exact_codes(x):
    """Nearest e4m3 values of x, ties to the even code, by a search among all of them."""
    every = _exact_e4m3()[:127]                                # the positive ones, ascending
    mag = x.abs().clamp(max=448).contiguous()
    hi = torch.searchsorted(every, mag).clamp(1, 126)
    a, b = every[hi - 1], every[hi]
    up = (mag - a > b - mag) | ((mag - a == b - mag) & (hi % 2 == 0))
    return torch.where(up, b, a).copysign(x)


def _exact_scale(amax):
    s = 2.0 ** -80
    while 448 * s < amax and s < 256:
        s *= 2
    return s


def exact(case, seed):
    if case["op"] == "select":
        return None
    st = prepare(case, seed)
    if case["op"] == "axes":
        n, d = case["tokens"], case["d"]
        a = torch.stack([st["positions"][:, int(x)].double() * f for x, f in zip(st["axes"].tolist(), st["inv_freq"].double())], -1)
        turn = torch.polar(torch.ones_like(a), a)[:, None]

        def one(x, w, b):
            x = x.double()
            if case["norm"] == "layer":
                x = (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + 1e-6)
            elif case["norm"] == "rms":
                x = x * torch.rsqrt((x * x).sum(-1, keepdim=True) / d + 1e-6)
            x = x * w.double() if w is not None else x
            x = x + b.double() if b is not None else x
            x = x.view(n, -1, d // 2, 2) if case["rope"] == "pairs" else x.view(n, -1, 2, d // 2).transpose(2, 3)
            y = torch.view_as_real(torch.complex(x[..., 0], x[..., 1]) * turn)
            return (y if case["rope"] == "pairs" else y.transpose(2, 3)).reshape(n, -1, d)

        return one(st["q"], st["qw"], st["qb"]), one(st["k"], st["kw"], st["kb"]), st["v"].double()
    hkv, d = case["kv_heads"], case["d"]
    cached, new = _lengths(case)
    cu = [0] + [int(x) for x in np.cumsum(new)]
    table = st["table"].tolist()
    if case["op"] == "append8":
        if sum(-(-m // PAGE) + 1 for m in new) * hkv > 20000:
            return None
        outs = [[], []]
        for s, (c, m) in enumerate(zip(cached, new)):
            start = c // PAGE * PAGE
            rec = st["pages"][table[s][start // PAGE]]
            for i, x in enumerate((st["k"], st["v"])):
                x = x[cu[s]:cu[s + 1]].double().clamp(-65504, 65504)
                before = _exact_record(rec, d)[i][:, :c - start].transpose(0, 1)
                y, parts = torch.cat([before, x]), []
                for p in range(0, y.shape[0], PAGE):
                    fresh = y[max(p, c - start):p + PAGE].abs().amax((0, 2)).tolist()
                    scale = torch.tensor([_exact_scale(f) for f in fresh], dtype=torch.float64, device=y.device)
                    if p < c - start:
                        scale = torch.maximum(scale, rec[:, 64 * d:64 * d + 8].contiguous().view(torch.float32)[:, i].double())
                    parts.append(_exact_codes(y[p:p + PAGE] / scale[:, None]) * scale[:, None])
                z = torch.cat(parts)
                outs[i].append(z.clamp(-65504, 65504) if case["dtype"] == "fp16" else z)
        return [torch.cat(o) for o in outs]
    group = case["q_heads"] // hkv
    outs = []
    if case["op"] == "selected":
        sel, seqs, positions = st["selected"].cpu().numpy(), st["token_seq"].tolist(), st["positions"].tolist()
        for t in range(len(seqs)):
            for h in range(hkv):
                pages = sel[t, h][sel[t, h] >= 0]
                k, v = _exact_record(st["pages"][[table[seqs[t]][p] for p in pages], h], d)
                at = torch.as_tensor(pages, device="cuda")[:, None] * PAGE + torch.arange(PAGE, device="cuda")
                keep = (at <= positions[t]).view(-1)
                w = torch.softmax(st["q"][t, h * group:(h + 1) * group].double() @ k.view(-1, d)[keep].T / math.sqrt(d), -1)
                outs.append(w @ v.view(-1, d)[keep])
        return torch.stack(outs).view(len(seqs), case["q_heads"], d)
    for s, (c, m) in enumerate(zip(cached, new)):
        end = c + m
        k, v = _exact_record(st["pages"][st["table"][s, :-(-end // PAGE)].long()], d)              # [pages, hkv, 64, d]
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
