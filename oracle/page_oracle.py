"""Plain numpy statement, in float64, of the operators over a shared pool of 4-bit pages: the quantiser with fp16
parameters rounded outwards, the page record, the step's bookkeeping, append, ragged causal attention, and the norm with
rotation.  Test infrastructure only; written from the definitions, one sequence and one head at a time."""
from __future__ import annotations

import numpy as np

PAGE = 64
_HALVES = np.sort(np.arange(65536, dtype=np.uint16).view(np.float16)[np.isfinite(np.arange(65536, dtype=np.uint16).view(np.float16))].astype(np.float64))


def half_down(x):
    """Largest finite float16 not above x (x inside +-65504)."""
    return _HALVES[np.searchsorted(_HALVES, x, side="right") - 1]


def half_up(x):
    return _HALVES[np.searchsorted(_HALVES, x, side="left")]


def quantise(x, axis):
    """(codes, scale, offset) of 4-bit groups along `axis`, the parameters with that axis kept."""
    x = np.clip(np.asarray(x, np.float64), -65504, 65504)
    z = half_down(x.min(axis, keepdims=True))
    s = half_up((x.max(axis, keepdims=True) - z) / 15)
    s = np.where(15 * s + z > 65504, _HALVES[np.searchsorted(_HALVES, s) - 1], s)      # no code stands for more than 65504
    s = np.where(s == 0, 1.0, s)
    return np.clip(np.rint((x - z) / s), 0, 15).astype(np.int64), s, z


def key_place(tok, ch):
    """(byte in the record, shift) of the key code of a token and channel, record of head_dim d."""
    return (ch // 32 * 2 + ch % 8 // 4) * 512 + (tok % 8) * 64 + (ch % 32 // 8) * 16 + (tok // 16) * 4 + (ch % 2) * 2 + ch % 4 // 2, tok // 8 % 2 * 4


def value_place(tok, ch, d):
    return 32 * d + (tok // 16) * 8 * d + (ch // 64) * 512 + (ch % 64 // 8) * 64 + (tok % 8 // 2) * 16 + (ch % 8 // 2) * 4 + (tok % 2) * 2 + tok % 16 // 8, ch % 2 * 4


def read_record(rec, d):
    """Keys and values (float64 [64, d]) of one record (uint8 [72 d])."""
    tok, ch = np.arange(PAGE)[:, None], np.arange(d)[None, :]
    kb, ks = key_place(tok, ch)
    vb, vs = value_place(tok, ch, d)
    with np.errstate(invalid="ignore"):
        par = rec[64 * d:].copy().view(np.float16).astype(np.float64)
    at = ch // 64 * PAGE + tok % 8 * 8 + tok // 8
    k = (rec[kb] >> ks & 15) * par[None, :d] + par[None, d:2 * d]
    v = (rec[vb] >> vs & 15) * par[2 * d + at] + par[3 * d + at]
    return k, v


class Sequence:
    """What one sequence's pages hold for one head, grown token by token."""

    def __init__(self, d):
        self.d, self.k, self.v = d, np.zeros((0, d)), np.zeros((0, d))

    def append(self, k, v):
        k, v = np.asarray(k, np.float64), np.asarray(v, np.float64)
        c, s, z = quantise(v.reshape(len(v), self.d // 64, 64), -1)
        self.v = np.concatenate([self.v, (c * s + z).reshape(len(v), self.d)])
        done = len(self.k) // PAGE * PAGE
        self.k = np.concatenate([self.k, k])
        for p in range(done, len(self.k) // PAGE * PAGE, PAGE):
            c, s, z = quantise(self.k[p:p + PAGE], 0)
            self.k[p:p + PAGE] = c * s + z


def attention(q, k, v, scale, window=0):
    """q [m, d]: the last m tokens of a sequence that holds keys k, values v [n, d]; float64."""
    m, n = len(q), len(k)
    out = np.zeros((m, v.shape[1] if n else q.shape[1]))
    for i in range(m):
        at = n - m + i
        lo = max(0, at - window + 1) if window else 0
        if at < 0:
            continue
        w = k[lo:at + 1] @ q[i] * scale
        w = np.exp(w - w.max())
        out[i] = w @ v[lo:at + 1] / w.sum()
    return out


def norm_rope(x, norm, w, b, eps, rope, rotary, inv_freq, pos):
    """x [n, heads, d] float64."""
    x = np.asarray(x, np.float64)
    n, h, d = x.shape
    if norm == "layer":
        x = (x - x.mean(-1, keepdims=True)) / np.sqrt(x.var(-1, keepdims=True) + eps)
    elif norm == "rms":
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if norm is not None:
        x = x * (1 if w is None else w) + (0 if b is None else b)
    y = x.copy()

    def turn(lo, hi, at, f):               # channel indices lo[i], hi[i] turn by at * inv_freq[f[i]]
        a = np.asarray(at, np.float64)[:, None] * np.asarray(inv_freq, np.float64)[f][None, :]
        c, s = np.cos(a)[:, None], np.sin(a)[:, None]
        y[..., lo] = x[..., lo] * c - x[..., hi] * s
        y[..., hi] = x[..., hi] * c + x[..., lo] * s

    if rope == "half":
        i = np.arange(rotary // 2)
        turn(i, i + rotary // 2, pos, i)
    elif rope == "pairs":
        i = np.arange(rotary // 2)
        turn(2 * i, 2 * i + 1, pos, i)
    elif rope == "2d":
        i = np.arange(d // 4)
        for part in (0, 1):
            turn(part * d // 2 + i, part * d // 2 + d // 4 + i, pos[:, part], i)
    return y


def plan(cached, new, table, ring, state, max_tokens):
    """The step's bookkeeping, sequence by sequence; table and ring are updated in place.  Returns (state, cu, total,
    slot, seq, pos)."""
    n_pages, width = len(ring), table.shape[1]
    head, left = int(state[0]) % n_pages, int(state[1])
    free = head + left
    cu, total, slot, seq, pos, refused, short = [0], [], [], [], [], 0, False
    for s, (c, m) in enumerate(zip(cached, new)):
        c, m = max(0, int(c)), int(m)
        have = -(-c // PAGE)
        if m < 0:
            for b in range(min(have, width)):
                ring[free % n_pages] = table[s, b]
                free += 1
            cu.append(cu[-1])
            total.append(0)
            continue
        need = -(-(c + m) // PAGE) - have
        ok = have + need <= width and (m == 0 or cu[-1] + m <= max_tokens)
        if ok and need > 0 and (short or need > left):
            ok, short = False, True
        if ok:
            for b in range(need):
                table[s, have + b] = ring[head % n_pages]
                head, left = head + 1, left - 1
        refused += not ok
        for i in range(c, c + m):
            slot.append(int(table[s, i // PAGE]) * PAGE + i % PAGE if ok else -1)
            seq.append(s)
            pos.append(i)
        cu.append(cu[-1] + m)
        total.append(c + m if ok else c)
    live = min(len(slot), max_tokens)
    pad = max_tokens - live
    arr = lambda x: np.asarray(x, np.int64).astype(np.int32)  # noqa: E731
    return (arr([head % n_pages, left + (free - int(state[0]) % n_pages - int(state[1])), refused, live]),
            np.minimum(arr(cu), max_tokens), arr(total), arr(slot[:live] + [-1] * pad), arr(seq[:live] + [-1] * pad),
            arr(pos[:live] + [0] * pad))
