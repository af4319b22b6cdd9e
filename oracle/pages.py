"""Paged 8-bit K/V store in float64 NumPy: quantisation, append, read and attention.

A page holds 64 positions.  Per page, layer, K/V head and side (keys, values) it has e4m3
codes and one power-of-two scale; a code c stands for value(c) * scale.  e4m3 (the OCP 8-bit
float without infinities): sign, 4 exponent bits of bias 7, 3 mantissa bits, subnormals at
exponent 0, the code 0x7f / 0xff NaN, largest value 448.
"""
import numpy as np

PAGE = 64
E_MIN, E_MAX = -110, 120
LAST = 240.0  # the largest code value at the scale 2^E_MAX: the next would stand for 2^128


def _positive():
    """Values of the codes 0 .. 0x7e, ascending."""
    out = []
    for c in range(0x7f):
        e, m = c >> 3, c & 7
        out.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return np.array(out)


POSITIVE = _positive()
VALUES = np.concatenate([POSITIVE, [np.nan], -POSITIVE, [np.nan]])


def encode(y):
    """Nearest e4m3 code of y (float64 array, |y| <= 448 where finite), ties to the even code;
    NaN code for values that are not finite."""
    y = np.asarray(y, dtype=np.float64)
    finite = np.isfinite(y)
    a = np.where(finite, np.abs(y), 0.0)
    hi = np.clip(np.searchsorted(POSITIVE, a), 0, 0x7e)  # the first value >= a
    lo = np.maximum(hi - 1, 0)
    up, down = POSITIVE[hi] - a, a - POSITIVE[lo]
    code = np.where(up < down, hi, np.where(up > down, lo, np.where(hi % 2 == 0, hi, lo)))
    code = np.where(POSITIVE[hi] == a, hi, code)
    return np.where(finite, code + 0x80 * np.signbit(y), 0x7f).astype(np.uint8)


def decode(codes):
    return VALUES[codes]


def scale_of(x):
    """2^e of the least e in [E_MIN, E_MAX] with max finite |x| <= 448 2^e (0: E_MIN)."""
    a = np.abs(np.asarray(x, dtype=np.float64))
    a = a[np.isfinite(a)]
    top = a.max() if a.size else 0.0
    e = E_MIN
    while e < E_MAX and top > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


class Pages:
    """codes uint8 [n_pages, n_layers, Hkv, 2, 64 dh] and scales float64 [n_pages, n_layers, Hkv, 2], in place."""

    def __init__(self, codes, scales):
        self.codes, self.scales = codes, scales
        self.n_pages, self.n_layers, self.heads, _, w = codes.shape
        self.dh = w // PAGE

    def side(self, page, layer, h, s):
        """Codes of one side as a [64, dh] view."""
        c = self.codes[page, layer, h, s]
        return c.reshape(PAGE, self.dh) if s == 0 else c.reshape(self.dh, PAGE).T

    def append(self, layer, ids, length, k, v):
        """Row with pages ids: its positions [length, length + n) take k, v [Hkv, n, dh]."""
        n = min(k.shape[1], len(ids) * PAGE - length)
        for i in range(length // PAGE, -(-(length + n) // PAGE) if n > 0 else 0):
            page, lo, hi = ids[i], max(length, i * PAGE), min(length + n, (i + 1) * PAGE)
            if not 0 <= page < self.n_pages:
                continue
            a, b = lo - i * PAGE, hi - i * PAGE
            for h in range(self.heads):
                for s, x in ((0, k), (1, v)):
                    new = np.asarray(x[h, lo - length:hi - length], dtype=np.float64)
                    scale, old = scale_of(new), self.scales[page, layer, h, s]
                    at = self.side(page, layer, h, s)
                    if a > 0:
                        if scale > old:
                            at[:a] = encode(decode(at[:a]) * (old / scale))
                        scale = max(scale, old)
                    with np.errstate(invalid="ignore"):
                        y = new / scale
                        if scale == 2.0 ** E_MAX:
                            y = np.where(np.isfinite(y), np.clip(y, -LAST, LAST), y)
                        at[a:b] = encode(y)
                    self.scales[page, layer, h, s] = scale

    def read(self, layer, ids, length):
        """(k, v) [Hkv, length, dh] and which positions are on present pages."""
        k, v = np.zeros((2, self.heads, length, self.dh))
        there = np.zeros(length, dtype=bool)
        for i in range(-(-length // PAGE)):
            if 0 <= ids[i] < self.n_pages:
                a, m = i * PAGE, min(PAGE, length - i * PAGE)
                there[a:a + m] = True
                for h in range(self.heads):
                    for s, x in ((0, k), (1, v)):
                        x[h, a:a + m] = decode(self.side(ids[i], layer, h, s)[:m]) * self.scales[ids[i], layer, h, s]
        return k, v, there


def attend(q, k, v):
    """q [H, n, dh] over k, v [Hkv, keys, dh]: (o [n, H, dh], lse [H, n]); 0 and -inf without keys."""
    H, n, dh = q.shape
    G = H // k.shape[0]
    o, lse = np.zeros((n, H, dh)), np.full((H, n), -np.inf)
    if k.shape[1] == 0:
        return o, lse
    for h in range(H):
        s = q[h].astype(np.float64) @ k[h // G].T / np.sqrt(dh)
        top = s.max(axis=1, keepdims=True)
        e = np.exp(s - top)
        total = e.sum(axis=1, keepdims=True)
        o[:, h] = (e / total) @ v[h // G]
        lse[h] = (top + np.log(total))[:, 0]
    return o, lse


def _up(x):
    return -(-x // PAGE)


def assign(table, lens, news, ids, free, size):
    """Pages of a stack (ids[:free], taken from the back) for the positions [len, len + new) of the rows of
    table, in place: (tokens granted to each row, their slots per row, free pages left)."""
    left, granted, slots = free, [], []
    waiting = False  # a row that does not get its pages stops those behind it that need some
    for row, length, new in zip(table, lens, news):
        if length + new > len(row) * PAGE:
            new = 0
        need = range(_up(length), _up(length + new))
        waiting = waiting or len(need) > left
        if len(need) and waiting:
            new, need = 0, ()
        for e in need:
            left -= 1
            row[e] = ids[left]
        granted.append(new)
        pages = [row[p // PAGE] for p in range(length, length + new)]
        slots.append([g * PAGE + p % PAGE if 0 <= g < size else -1 for g, p in zip(pages, range(length, length + new))])
    return granted, slots, left


def release(table, lens, news, ids, free, size):
    """The pages of the positions [len, len + new) of each row back onto the stack: free pages after it."""
    for row, length, new in zip(table, lens, news):
        if length + new > len(row) * PAGE:
            continue
        for e in range(_up(length), _up(length + new)):
            if 0 <= row[e] < size:
                ids[free] = row[e]
                free += 1
            row[e] = -1
    return free


def groups(table, lens, min_pages=1):
    """(first row of each row's group, pages that the group shares): neighbours with min_pages or more whole
    leading pages in common stand in one group, which shares what all of them do; 0 for a row alone."""
    lead, shared = [], [0] * len(table)
    for b, row in enumerate(table):
        common = 0
        while b and common < min(lens[b], lens[b - 1]) // PAGE and row[common] == table[b - 1][common]:
            common += 1
        if b and common >= min_pages:
            lead.append(lead[-1])
            shared[lead[b]] = min(shared[lead[b]], common) if shared[lead[b]] else common
        else:
            lead.append(b)
    return lead, [shared[a] for a in lead]
