"""fp64 oracle of serving from a committed cache of 8 bits: page tables and slot
maps from request lengths, rows into the cache, and what the cache holds.  TEST
INFRASTRUCTURE ONLY; it shares no code with the HIP path.

The cache holds, per (layer, page, head), e4m3 codes of 16 keys and of 16 values
and a scale byte b for each: an entry is code * 2^(b - 127).  Everything here is
loops over pages and sequences, in float64 and Python integers.
"""
from __future__ import annotations

import math

import numpy as np

from . import PAGE, SKIP

OK, ERR_CAPACITY, ERR_PAGE_RANGE, ERR_LENGTH, ERR_POOL = 0, 4, 5, 7, 10


# --------------------------------------------------------------------- codes

def e4m3_values():
    """The value of every code: sign, 4 exponent bits (bias 7), 3 bits of fraction; codes
    0x7F and 0xFF are NaN, there is no infinity."""
    out = np.empty(256)
    for c in range(256):
        sign, e, m = -1.0 if c & 128 else 1.0, (c >> 3) & 15, c & 7
        if e == 15 and m == 7:
            out[c] = math.nan
        else:
            out[c] = sign * (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return out


VALUES = e4m3_values()
_POSITIVE = VALUES[:127]            # codes 0 .. 0x7E, ascending


def e4m3_code(x):
    """Nearest code of |x| <= 448, ties to the even one; anything not finite is NaN."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    hi = np.searchsorted(_POSITIVE, a).clip(0, 126)      # first value >= a
    lo = np.maximum(hi - 1, 0)
    up, down = _POSITIVE[hi] - a, a - _POSITIVE[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = code | np.where(np.signbit(x), 128, 0)
    return np.where(np.isfinite(x), code, 127).astype(np.uint8)


def scale_byte(rows):
    """b of the smallest 2^(b - 127) >= max |x| / 448 over the finite entries; at least 1."""
    a = np.abs(np.asarray(rows, np.float64))
    top = np.where(np.isfinite(a), a, 0.0).max(initial=0.0)
    if top == 0.0:
        return 1
    m, e = math.frexp(top)                               # top = 2m * 2^(e - 1), 2m in [1, 2)
    return max(1, e - 9 + (1 if 2 * m > 1.75 else 0) + 127)


# --------------------------------------------------------------------- cache

class Cache8:
    """Codes k, v [L][pages][Hkv][16][hd] (the values' too: token major here) and scale bytes."""

    def __init__(self, k, v, ks, vs):
        self.k, self.v, self.ks, self.vs = (np.array(x) for x in (k, v, ks, vs))

    @classmethod
    def read(cls, t):
        """From the library's uint8 tensors."""
        c = {k: x.cpu().numpy() for k, x in t.items()}
        return cls(c["k_pages"], c["v_pages"].swapaxes(3, 4), c["k_scale"], c["v_scale"])

    def values(self, which, layer, page, g):
        codes, b = (self.k, self.ks) if which == "k" else (self.v, self.vs)
        return VALUES[codes[layer, page, g]] * 2.0 ** (int(b[layer, page, g]) - 127)

    def store(self, rows_k, rows_v, row_dst, num_pages):
        """Rows [L][M][Hkv][hd] to the slots row_dst.  Returns the status."""
        status, runs = OK, []
        for r, d in enumerate(int(x) for x in row_dst):
            if d < 0:
                continue
            if d // PAGE >= num_pages:
                status = status or ERR_PAGE_RANGE
            elif runs and runs[-1][-1] == (r - 1, d - 1) and d % PAGE:
                runs[-1].append((r, d))
            else:
                runs.append([(r, d)])
        for run in runs:
            page, t0, n, r0 = run[0][1] // PAGE, run[0][1] % PAGE, len(run), run[0][0]
            for rows, codes, scale in ((rows_k, self.k, self.ks), (rows_v, self.v, self.vs)):
                for layer in range(codes.shape[0]):
                    for g in range(codes.shape[2]):
                        x = np.asarray(rows[layer, r0:r0 + n, g], np.float64)
                        self._page(codes[layer, page, g], scale, (layer, page, g), x, t0)
        return status

    @staticmethod
    def _page(codes, scale, at, x, t0):
        b = scale_byte(x)
        if t0 == 0:
            codes[:] = 0
        else:
            old = int(scale[at])
            b = max(b, old)
            if b > old:
                codes[:] = e4m3_code(VALUES[codes] * 2.0 ** (old - b))
        codes[t0:t0 + len(x)] = e4m3_code(x * 2.0 ** (127 - b))
        scale[at] = b

    def context(self, table, s, layer, g, n):
        """Keys and values [n][hd] of sequence s's first n positions."""
        pages = [int(table[s][p]) for p in range(-(-n // PAGE))]
        hd = self.k.shape[4]
        cat = lambda w: (np.concatenate([self.values(w, layer, p, g) for p in pages])  # noqa: E731
                         if pages else np.zeros((0, hd)))[:n]
        return cat("k"), cat("v")


# -------------------------------------------------------------- pages and slots

def assign_pages(want, reserve, table, held, free, max_pages, num_pages):
    """Pages of lengths want: (table, held, free list, status) afterwards; ``free`` is the
    list of free pages.  Works page by page through the numbering of the definition."""
    table, held, free, status = np.array(table), list(map(int, held)), list(free), OK
    need = []
    for s, w in enumerate(int(x) for x in want):
        n = -(-(w + reserve) // PAGE) if w > 0 else 0
        err = (ERR_LENGTH if held[s] < 0 or held[s] > max_pages or w < 0
               else ERR_CAPACITY if n > max_pages else OK)
        status = status or err
        need.append(held[s] if err else n)
    released = [(s, p) for s in range(len(need)) for p in range(need[s], held[s])]
    room = len(free) + len(released)
    if room > num_pages:                 # holdings that the pool cannot have
        return table, held, free, status or ERR_POOL
    places, asked = [], 0
    for s in range(len(need)):
        grow = max(0, need[s] - held[s])
        asked += grow
        if grow and asked > room:
            status = status or ERR_POOL
            need[s] = held[s]
        elif grow:
            places += [(s, p) for p in range(held[s], need[s])]
    pages = [int(table[s][p]) for s, p in released]
    for s, p in released:
        table[s][p] = -1
    for k, (s, p) in enumerate(places):
        table[s][p] = pages[k] if k < len(pages) else free[len(free) + len(pages) - 1 - k]
    if len(places) >= len(pages):
        free = free[:len(free) - (len(places) - len(pages))]
    else:
        free = free + pages[len(places):][::-1]
    moved = pages + [int(table[s][p]) for s, p in places]
    if any(not 0 <= x < num_pages for x in moved):
        status = status or ERR_PAGE_RANGE
    return table, need, free, status


def slot_map(num_rows, row_start, pos0, table, max_pages, num_pages):
    """(row_pos, row_dst, status) of packed rows."""
    pos, dst, status = np.zeros(num_rows, np.int32), np.full(num_rows, SKIP, np.int32), OK
    if any(int(a) > int(b) for a, b in zip(row_start, row_start[1:])):
        return pos, dst, ERR_LENGTH      # which row is whose is not defined
    for s in range(len(pos0)):
        for r in range(int(row_start[s]), min(num_rows, int(row_start[s + 1]))):
            p = int(pos0[s]) + r - int(row_start[s])
            page = int(table[s][p // PAGE]) if 0 <= p < max_pages * PAGE else -1
            err = (ERR_LENGTH if pos0[s] < 0 else ERR_CAPACITY if p >= max_pages * PAGE
                   else ERR_PAGE_RANGE if not 0 <= page < num_pages else OK)
            status = status or err
            if not err:
                pos[r], dst[r] = p, page * PAGE + p % PAGE
    return pos, dst, status
