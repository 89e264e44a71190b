"""64-bit reference of the paged cache in 8 bits and of the pages' bookkeeping (numpy, plain loops)."""
import math

import numpy as np

from .paged import rotate

LEAST = -100   # exponent of the least scale


def _values():
    out = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[c] = math.nan if c & 127 == 127 else -x if c & 128 else x
    return out


VALUES = _values()                       # what each code stands for
_POSITIVE = VALUES[:127]                 # ascending


def encode(x):
    """The nearest codes of finite x with |x| <= 448, ties to the even code; not finite: 0x7f (a NaN's sign is not looked at)."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    hi = np.searchsorted(_POSITIVE, a).clip(max=126)
    lo = (hi - 1).clip(min=0)
    d = (a - _POSITIVE[lo]) - (_POSITIVE[hi] - a)
    code = np.where((d < 0) | ((d == 0) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.isfinite(x), code | np.where(np.signbit(x), 128, 0), 127)
    return code.astype(np.uint8)


def scale_of(top):
    """The least power of two that takes top to 448 or below, 2^LEAST at the least."""
    if not top > 0:
        return 2.0 ** LEAST
    m, e = math.frexp(top)
    return 2.0 ** max(LEAST, e - 8 if m > 0.875 else e - 9)


def append(codes, scales, table, lens, start, page, block, rows, theta=None, dim=0):
    """codes [pages][page][heads][dh] uint8 and scales [pages][blocks][heads] (changed in place) after rows [n][heads][dh] were
    appended, rotated with theta. Returns the exact values [n][heads][dh] before their rounding and each row's scales [n][heads]."""
    exact = np.zeros(rows.shape)
    used = np.zeros(rows.shape[:2])
    for b in range(len(lens)):
        lo, hi = int(start[b]), int(start[b + 1])
        p0 = int(lens[b]) - (hi - lo)
        blocks = {}
        for t in range(lo, hi):
            pos = p0 + t - lo
            blocks.setdefault((pos // page, pos % page // block), []).append((t, pos))
            exact[t] = rows[t] if theta is None else rotate(rows[t], pos, theta, dim)
        for (i, sub), members in blocks.items():
            pg = int(table[b, i])
            raw = np.abs(rows[[t for t, _ in members]])
            top = np.where(np.isfinite(raw), raw, 0.0).max(axis=(0, 2)) * (1.0 if theta is None else 2.0)
            fresh = np.array([scale_of(x) for x in top])
            first = members[0][1]
            s0 = sub * block
            if first % page > s0:
                before = scales[pg, sub].copy()
                fresh = np.maximum(fresh, 2.0 ** np.ceil(np.log2(before)))   # powers of two, whatever the earlier tokens came with
                at = slice(s0, first % page)
                grown = fresh != before
                old = VALUES[codes[pg, at]] * before[None, :, None]
                codes[pg, at] = np.where(grown[None, :, None], encode(old / fresh[None, :, None]), codes[pg, at])
            scales[pg, sub] = fresh
            for t, pos in members:
                used[t] = fresh
                codes[pg, pos % page] = encode(exact[t] / fresh[:, None])
    return exact, used


def resize(ring, state, table, lens, want, page, rows):
    """The pages' bookkeeping, sequence after sequence: (ring, state, table, lens, start, [(slot, sequence, position)], found), all new.
    found: "no room", "bad sequence", "bad page" (-1, no page, apart), "bad pool"."""
    ring, table, out = ring.copy(), table.copy(), np.array(lens).copy()
    n, width = len(ring), table.shape[1]
    first, count = (int(x) for x in state)
    free = [int(ring[(first + i) % n]) for i in range(count)]
    taken, back, made, start, found = 0, [], [], [0], set()
    asked_pages = asked_rows = 0
    for b in range(len(out)):
        have, shall = int(lens[b]), int(want[b])
        if not (0 <= have <= width * page and 0 <= shall <= width * page):
            found.add("bad sequence")
        elif shall > have:
            held, needed = -(-have // page), -(-shall // page)
            asked_pages += needed - held
            asked_rows += shall - have
            if (needed > held and asked_pages > count) or asked_rows > rows:
                found.add("no room")
            else:
                table[b, held:needed] = free[taken:taken + needed - held]
                if any(not 0 <= x < n for x in free[taken:taken + needed - held]):
                    found.add("bad page")
                taken += needed - held
                out[b] = shall
                made += [(int(table[b, p // page]) * page + p % page, b, p) for p in range(have, shall)]
        else:
            given = [int(x) for x in table[b, -(-shall // page):-(-have // page)]]
            back += [x for x in given if 0 <= x < n]
            if any(x >= n or x < -1 for x in given):
                found.add("bad page")
            out[b] = shall
        start.append(len(made))
    if len(back) > n - count:
        found.add("bad pool")
        back = back[:n - count]
    for i, p in enumerate(back):
        ring[(first + count + i) % n] = p
    return ring, ((first + taken) % n, count - taken + len(back)), table, out, start, made, found
