"""Plain numpy statement, in float64, of the operators over a shared pool of 8-bit pages: the e4m3 quantiser with one
power-of-two scale a page, the page record, appends that raise the scale, the mean key, the selection of pages, attention over
a selection, and the rotation by several positions a token.  Test infrastructure only; written from the definitions, one
sequence and one head at a time."""
from __future__ import annotations

import numpy as np

PAGE = 64


def e4m3_values():
    """The value of every code (NaN for 127 and 255)."""
    out = []
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v = np.nan if c & 127 == 127 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out.append(-v if c > 127 else v)
    return np.array(out)


VALUES = e4m3_values()
_POSITIVE = VALUES[:127]                    # ascending, index = code


def nearest(x):
    """The e4m3 values nearest to x, ties to the even code, beyond 448 the largest."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 1, 126)
    lo = hi - 1
    dl, dh = a - _POSITIVE[lo], _POSITIVE[hi] - a
    up = (dh < dl) | ((dh == dl) & (hi % 2 == 0))
    return np.where(up, _POSITIVE[hi], _POSITIVE[lo]) * np.where(np.signbit(x), -1.0, 1.0)


def exponent(amax):
    """The smallest e in [-80, 8] with 448 * 2^e >= amax."""
    e = -80
    while e < 8 and 448.0 * 2.0 ** e < amax:
        e += 1
    return e


def key_place(tok, ch, d):
    """Byte in the record of the key code of a token and channel."""
    return (tok // 8 * (d // 64) + ch // 64) * 512 + tok % 8 * 64 + ch % 64


def value_place(tok, ch, d):
    w = d // 8
    return 64 * d + 32 + ((tok // 16 * 2 + tok // 8 % 2) * 2 + tok % 2) * 32 * w + (ch // w * 4 + tok % 8 // 2) * w + ch % w


def read_record(rec, d):
    """Key codes and value codes (their values, float64 [64, d]), scales, factor and mean codes of one record (uint8 [130 d])."""
    tok, ch = np.arange(PAGE)[:, None], np.arange(d)[None, :]
    par = rec[64 * d:64 * d + 12].copy().view(np.float32).astype(np.float64)
    return (VALUES[rec[key_place(tok, ch, d)]], VALUES[rec[value_place(tok, ch, d)]], par[0], par[1], par[2],
            rec[128 * d + 32:129 * d + 32].copy().view(np.int8).astype(np.int64))


class Block:
    """The keys or values of one page, grown by appends."""

    def __init__(self, d):
        self.codes, self.e = np.zeros((0, d)), -80

    def append(self, x):
        x = np.clip(np.asarray(x, np.float64), -65504, 65504)
        e = max(exponent(np.abs(x).max(initial=0.0)), self.e if len(self.codes) else -80)
        old = nearest(self.codes * 2.0 ** (self.e - e)) if e > self.e else self.codes
        self.codes, self.e = np.concatenate([old, nearest(x / 2.0 ** e)]), e

    def values(self):
        return self.codes * 2.0 ** self.e


class Sequence:
    """What one sequence's pages hold for one head, an append (of one call) at a time."""

    def __init__(self, d):
        self.d, self.blocks, self.n = d, [], 0

    def append(self, k, v):
        k, v, at = np.asarray(k, np.float64), np.asarray(v, np.float64), 0
        while at < len(k):
            if self.n % PAGE == 0:
                self.blocks.append((Block(self.d), Block(self.d)))
            m = min(PAGE - self.n % PAGE, len(k) - at)
            self.blocks[-1][0].append(k[at:at + m])
            self.blocks[-1][1].append(v[at:at + m])
            self.n, at = self.n + m, at + m

    @property
    def k(self):
        return np.concatenate([b[0].values() for b in self.blocks]) if self.blocks else np.zeros((0, self.d))

    @property
    def v(self):
        return np.concatenate([b[1].values() for b in self.blocks]) if self.blocks else np.zeros((0, self.d))


def mean_key(codes, e):
    """(whole numbers [d], factor) of a full page's key codes."""
    s = codes.sum(0)                        # exact in float64, and a float32
    top = np.abs(s).max()
    if top == 0:
        return np.zeros(len(s), np.int64), 0.0
    inv = np.float32(127) / np.float32(top)
    return np.rint(s.astype(np.float32) * inv).astype(np.int64), float(top * 2.0 ** e / 64)


def scores(q, means):
    """float32 scores of pages with (codes, factor) for the query rows q [group, d] of one token."""
    best = np.full(len(means), -np.inf, np.float32)
    if not means:
        return best
    codes, factor = np.stack([m[0] for m in means]).astype(np.int64), np.array([m[1] for m in means], np.float32)
    for row in np.asarray(q, np.float32):
        a = np.maximum(np.abs(row).max(), np.float32(2.0 ** -60)).astype(np.float32)
        q8 = np.rint(row * (np.float32(127) / a)).astype(np.int64)
        best = np.maximum(best, (codes @ q8).astype(np.float32) * factor * a)
    return best


def select(q, means, mine, top, first, recent, there=None):
    """Pages that a token whose own page is `mine` selects; means[p] is None for a page that is not there, or not full (as the last
    may be); there[p]: whether it is there (None: all of the first and the most recent are)."""
    fixed = [p for p in range(mine + 1) if p < first or p > mine - recent]
    middle = [p for p in range(mine + 1) if p not in fixed and means[p] is not None]
    keep = [p for p in fixed if there is None or there[p]]
    s = scores(q, [means[p] for p in middle])
    order = sorted(range(len(middle)), key=lambda i: (-float(s[i]), middle[i]))
    out = sorted(keep + [middle[i] for i in order[:top - len(keep)]])
    return out + [-1] * (top - len(out))


def attention(q, k, v, scale):
    """q [group, d] of one token over the keys and values that it sees."""
    out = np.zeros((len(q), v.shape[1]))
    if len(k):
        w = q @ k.T * scale
        w = np.exp(w - w.max(-1, keepdims=True))
        out = w @ v / w.sum(-1, keepdims=True)
    return out


def rotate_axes(x, rope, inv_freq, pos, axes):
    """x [n, heads, d] float64 turned by pos [n, several], frequency i by the position axes[i]."""
    x, y = np.asarray(x, np.float64), np.array(x, np.float64)
    r = len(inv_freq)
    for i in range(r):
        lo, hi = (i, i + r) if rope == "half" else (2 * i, 2 * i + 1)
        if not 0 <= axes[i] < pos.shape[1]:
            continue
        a = pos[:, axes[i]].astype(np.float64) * float(inv_freq[i])
        c, s = np.cos(a)[:, None], np.sin(a)[:, None]
        y[..., lo] = x[..., lo] * c - x[..., hi] * s
        y[..., hi] = x[..., hi] * c + x[..., lo] * s
    return y
