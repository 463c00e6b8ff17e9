"""Definitions of the page plan and of the cache in pages of 8-bit numbers (numpy, host): e4m3 codes, the scale of a block,
rows written to and read from a paged cache, and the requests of a step served one after the other.  Attention over the
rows is that of paged_oracle, in double precision."""
from __future__ import annotations

import math

import numpy as np

NAN_CODE = 0x7f


def _value(code):
    sign, e, m = -1.0 if code & 0x80 else 1.0, (code >> 3) & 15, code & 7
    if e == 15 and m == 7:
        return math.nan
    return sign * (m / 8.0 * 2.0 ** -6 if e == 0 else (1.0 + m / 8.0) * 2.0 ** (e - 7))


VALUES = np.array([_value(c) for c in range(256)])                     # what each code stands for
_POSITIVE = VALUES[:127]                                                # ascending: codes 0 .. 126, 448 the last


def encode(x):
    """The nearest codes, ties to the even one; 448 at most in size; NaN stays."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.where(np.isnan(x), 0.0, np.abs(x)), 448.0)
    hi = np.searchsorted(_POSITIVE, a).clip(1, 126)                     # the first code that is not smaller
    lo = hi - 1
    below, above = a - _POSITIVE[lo], _POSITIVE[hi] - a
    code = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.isnan(x), NAN_CODE, code)
    return (code | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def scale_for(largest):
    """2^e, e the smallest integer from -126 to 120 with largest <= 448 * 2^e."""
    for e in range(-126, 120):
        if largest <= 448.0 * 2.0 ** e:
            return 2.0 ** e
    return 2.0 ** 120


def growth(magnitude):
    """What a rotation multiplies the largest number by at most, as the single-precision factor that enters the scale."""
    return float(max(np.float32(1.0), np.float32(math.sqrt(2.0) * magnitude)))


def largest_of(x, factor=1.0):
    """factor * max |x| in single precision, NaN left out; x: the inputs of a block's new rows."""
    a = np.abs(np.asarray(x, dtype=np.float32))
    a = a[~np.isnan(a)]
    with np.errstate(over="ignore"):
        return float(a.max() * np.float32(factor)) if a.size else 0.0


class Cache:
    """Keys or values of a paged cache: codes [pages, heads, page, d] (uint8), scales [pages, heads, page / block] (float32)."""

    def __init__(self, codes, scales):
        self.codes, self.scales = codes.copy(), scales.copy()
        self.page = codes.shape[2]
        self.block = self.page // scales.shape[2]

    def place(self, table_row, row):
        """(page, row of the page), or None."""
        if row < 0 or row // self.page >= len(table_row):
            return None
        p = int(table_row[row // self.page])
        return (p, row % self.page) if 0 <= p < len(self.codes) else None

    def append(self, table_row, first, x, y, factor=1.0):
        """Rows first, first + 1, ...: y [n, heads, d] in double precision, the scale by the inputs x.  Returns which rows were
        written."""
        n, done, block = len(x), [], self.block
        for begin in range(first // block * block, first + n, block) if n else ():
            lo, hi = max(begin, first), min(begin + block, first + n)
            at = self.place(table_row, begin)
            if at is None:
                continue
            p, o = at
            for h in range(self.codes.shape[1]):
                s = scale_for(largest_of(x[lo - first:hi - first, h], factor))
                old = float(self.scales[p, h, o // block])
                if begin < first:
                    s = max(s, old)
                    if s > old:
                        rows = slice(o, o + first - begin)
                        self.codes[p, h, rows] = encode(VALUES[self.codes[p, h, rows]] * (old / s))
                self.scales[p, h, o // block] = s
                self.codes[p, h, o + lo - begin:o + hi - begin] = encode(y[lo - first:hi - first, h] / s)
            done += range(lo, hi)
        return done

    def rows(self, table_row, n, first=0):
        """([rows there, heads, d] in double precision, which rows those are) of rows first .. first + n - 1."""
        out, there = [], []
        for r in range(first, first + n):
            at = self.place(table_row, r)
            if at is not None:
                p, o = at
                out.append(VALUES[self.codes[p, :, o]] * self.scales[p, :, o // self.block, None].astype(np.float64))
                there.append(r)
        return np.stack(out) if out else np.zeros((0, self.codes.shape[1], self.codes.shape[3])), np.array(there, dtype=np.int64)


def plan(slots, new, table, seq_len, stack, n_free, page, n_pages, most):
    """The requests of a step, one after the other.  Returns a dict of what comes back, and the conditions met ("slot", "page",
    "room")."""
    table, seq_len, stack, said = table.copy(), seq_len.copy(), stack.copy(), set()
    cap = table.shape[1] * page
    seen, valid = set(), []
    for s in slots:
        ok = 0 <= s < len(table) and s not in seen
        if s != -1 and not ok:
            said.add("slot")
        if ok:
            seen.add(s)
        valid.append(ok)
    if not 0 <= n_free <= n_pages:
        said.add("page")
    free = min(max(n_free, 0), n_pages)
    for s, n, ok in zip(slots, new, valid):
        if ok and n < 0:
            for j in range(table.shape[1]):
                if 0 <= table[s, j] < n_pages:
                    if free < n_pages:
                        stack[free] = table[s, j]
                        free += 1
                    else:
                        said.add("page")
                table[s, j] = -1
            seq_len[s] = 0
    top, tokens, missing = free, 0, 0
    granted, first, cu, list_slots, list_rows = [], [], [0], [], []
    for s, n, ok in zip(slots, new, valid):
        got, length = 0, max(int(seq_len[s]), 0) if ok else 0
        if ok and n >= 0:
            if length + n > cap:
                said.add("page")
            else:
                want = [j for j in range(-(-length // page), -(-(length + n) // page)) if not 0 <= table[s, j] < n_pages]
                tokens, missing = tokens + n, missing + len(want)
                if tokens <= most and (not want or missing <= free):
                    got = n
                    for j in want:
                        top -= 1
                        table[s, j] = stack[top]
                else:
                    said.add("room")
        granted.append(got)
        first.append(length)
        cu.append(cu[-1] + got)
        list_slots += [s] * got
        list_rows += range(length, length + got)
    pad = most - len(list_slots)
    return dict(table=table, seq_len=seq_len, stack=stack, n_free=top, granted=granted, first=first, cu=cu,
                token_slots=list_slots + [-1] * pad, token_rows=list_rows + [0] * pad), said
