"""References of the paged 8-bit cache's operators (oracle side, test infrastructure).

Rotary positions and attention in float64; tables, slots, scales and codes
exactly, one request, row and element after the other.
"""
import numpy as np


def rope(x, positions, freqs, layout="half", scale=1.0, inverse=False):
    """x [n, H, d] -> float64, pairs of the first 2 len(freqs) elements turned."""
    y = np.array(x, dtype=np.float64)
    half = len(freqs)
    for i in range(half):
        a, b = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
        angle = np.asarray(positions, dtype=np.float64)[:, None] * freqs[i]
        c, s = np.cos(angle), np.sin(angle) * (-1.0 if inverse else 1.0)
        x0, x1 = y[:, :, a].copy(), y[:, :, b].copy()
        y[:, :, a] = scale * (x0 * c - x1 * s)
        y[:, :, b] = scale * (x1 * c + x0 * s)
    return y


def resize(table, lens, grow, page, n_pages, free, n_free, n_rows):
    """-> (table, free, new_lens, starts, slots, positions, new_free), the first two copies."""
    table, free = table.copy(), free.copy()
    n, max_pages = table.shape
    room, cap = max_pages * page, len(free)
    slots, positions = np.full(n_rows, -1, np.int64), np.full(n_rows, -1, np.int32)
    starts, ends, total = [0], [], 0
    for g in range(n):
        total += max(0, int(grow[g]))
        ends.append(total)
        starts.append(min(total, n_rows))
    good = [0 <= lens[g] <= room and 0 <= int(lens[g]) + int(grow[g]) <= room
            and ends[g] <= n_rows for g in range(n)]
    pages = lambda t: -(-int(t) // page)
    top = min(max(int(n_free), 0), cap)
    for g in range(n):
        if good[g]:
            for p in range(pages(lens[g] + grow[g]), pages(lens[g])):
                if top < cap:
                    free[top] = table[g, p]
                    top += 1
    asked, left = 0, top
    new_lens = np.full(n, -1, np.int32)
    for g in range(n):
        if not good[g]:
            continue
        have, want = pages(lens[g]), pages(lens[g] + grow[g])
        asked += max(0, want - have)
        if want > have and asked > top:
            continue
        for p in range(have, want):
            left -= 1
            table[g, p] = free[left]
        new_lens[g] = lens[g] + grow[g]
        for i in range(max(0, int(grow[g]))):
            r, at = starts[g] + i, int(lens[g]) + i
            positions[r] = at
            if 0 <= table[g, at // page] < n_pages:
                slots[r] = int(table[g, at // page]) * page + at % page
    return table, free, new_lens, np.array(starts, np.int32), slots, positions, left


def e4m3_values():
    """The values of the 256 codes (1-4-3, bias 7, no infinities)."""
    v = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[b] = -x if b & 128 else x
    v[[127, 255]] = np.nan
    return v


E4M3 = e4m3_values()


def code_values(codes, kind):
    """Bytes -> the numbers that they stand for (float64)."""
    return codes.view(np.int8).astype(np.float64) if kind == "int8" else E4M3[codes]


def to_codes(x, kind):
    """Nearest code to each of x (float64), ties to the even one."""
    if kind == "int8":
        return np.clip(np.rint(x), -127, 127).astype(np.int8).view(np.uint8)
    mag = E4M3[:127]
    a = np.abs(x)
    hi = np.clip(np.searchsorted(mag, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    below, above = a - mag[lo], mag[hi] - a
    code = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    code = np.where(a >= mag[126], 126, code)
    return (code + 128 * np.signbit(x)).astype(np.uint8)


def least_scale(amax, kind):
    """The least power of two, from 2^-126 on, that takes amax to the codes' range."""
    if amax == 0:
        return 0.0
    if not np.isfinite(amax):
        return np.nan
    e = -126
    while amax > (127.0 if kind == "int8" else 448.0) * 2.0 ** e:
        e += 1
    return 2.0 ** e


def write(x, slots, pages, scales, kind):
    """x [n, H, d] float32 into pages (bytes [n_pages, H, page, d]) and scales, both in place."""
    n_pages, H, page, _ = pages.shape
    r = 0
    slots = [int(s) if 0 <= s < n_pages * page else -1 for s in slots]
    while r < len(slots):
        if slots[r] < 0:
            r += 1
            continue
        end = r + 1
        while end < len(slots) and slots[end] > slots[end - 1] and slots[end] // page == slots[r] // page:
            end += 1
        p, first = slots[r] // page, slots[r] % page
        at = [s % page for s in slots[r:end]]
        for h in range(H):
            rows = np.asarray(x[r:end, h], dtype=np.float32)
            least = least_scale(float(np.abs(rows.astype(np.float64)).max()), kind)
            old = np.float32(scales[p, h]) if first else np.float32(0)
            new = np.float32(np.nan) if np.isnan(old) or np.isnan(least) else max(old, np.float32(least))
            if new > old:
                was = code_values(pages[p, h, :first], kind).astype(np.float32)
                pages[p, h, :first] = to_codes(((was * old) / new).astype(np.float64), kind)
            with np.errstate(all="ignore"):
                pages[p, h, at] = to_codes((rows / new).astype(np.float64), kind) if new > 0 else 0
            scales[p, h] = new
        r = end


def rows_of(pages, scales, table, length, h, kind):
    """The first `length` rows of head h of one sequence (float64), and whether all are known."""
    page = pages.shape[2]
    out = np.zeros((length, pages.shape[3]))
    for t in range(length):
        p = int(table[t // page])
        if not 0 <= p < pages.shape[0]:
            out[t] = np.nan
            continue
        out[t] = code_values(pages[p, h, t % page], kind) * float(scales[p, h])
    return out
