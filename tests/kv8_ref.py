"""Plain forms of the 8-bit cache's operators in 64 bits, written from their definitions (include/pasta_kv8.h): one request, block, row and head
after the other."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 16
TOP = {"e4m3": 448.0, "int8": 127.0}
E_MIN, E_MAX = -100, 119
UNUSED = -99


# ------------------------------------------------------------------------------------------------ codes
def code_values(codes):
    """value of each of the 256 bytes"""
    if codes == "int8":
        return np.arange(256, dtype=np.uint8).view(np.int8).astype(np.float64)
    out = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        v = math.nan if (b & 127) == 127 else m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out[b] = -v if b & 128 else v
    return out


def nearest(x, codes):
    """value of the code next to x, ties to even"""
    if codes == "int8":
        return np.clip(np.rint(x), -127, 127)
    grid = code_values("e4m3")[:127]
    a = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(grid, a), 1, 126)
    mid = (grid[hi - 1] + grid[hi]) / 2
    up = (a > mid) | ((a == mid) & (hi % 2 == 0))
    return np.copysign(np.where(up, grid[hi], grid[hi - 1]), x)


def exponent(amax, codes):
    e = E_MIN
    while e < E_MAX and amax > TOP[codes] * 2.0 ** e:
        e += 1
    return e


def k_natural(codes):
    """[..., D / 16, 16 tokens, 16] -> [..., 16 tokens, D]"""
    return np.moveaxis(codes, -2, -3).reshape(*codes.shape[:-3], BLOCK, -1)


def k_stored(x):
    return np.moveaxis(x.reshape(*x.shape[:-1], -1, 16), -2, -3)


# ------------------------------------------------------------------------------------------------ places
def slots(P, W, length, keep, offs, n_rows, table, stack, free):
    """(slot, length_out, free_out, table, stack) of a step, request by request"""
    table, stack, R = table.copy(), stack.copy(), len(length)
    kept = [min(length[r], keep[r]) if keep is not None else length[r] for r in range(R)]
    n = [offs[r + 1] - offs[r] for r in range(R)]
    old = [-(-int(length[r]) // P) for r in range(R)]
    new = [-(-int(kept[r] + n[r]) // P) for r in range(R)]
    fits = [kept[r] + n[r] <= W * P for r in range(R)]
    for r in range(R):
        for p in range(new[r], old[r]):
            if fits[r]:
                stack[free] = table[r, p]
                free += 1
    top, asked, taken = free, 0, 0
    slot, out = np.full(n_rows, -1), np.array(length)
    for r in range(R):
        need = max(0, new[r] - old[r]) if fits[r] else 0
        asked += need
        if not fits[r] or (need and asked > top):
            continue
        for p in range(old[r], new[r]):
            table[r, p] = stack[top - 1 - taken]
            taken += 1
        out[r] = kept[r] + n[r]
        for i in range(n[r]):
            t = kept[r] + i
            slot[offs[r] + i] = table[r, t // P] * P + t % P
    return slot, out, top - taken, table, stack


# ------------------------------------------------------------------------------------------------ rows
def append(codes, values, scale, new, slot, P):
    """Values (natural order [pages, H, B, 16, D]) and scales [pages, H, B] after rows new [n, H, D] went to the slots; both are changed in place."""
    i, n_slots = 0, values.shape[0] * P
    while i < len(slot):
        if not 0 <= slot[i] < n_slots:
            i += 1
            continue
        j = i + 1
        while j < len(slot) and slot[j] == slot[j - 1] + 1 and slot[j] // BLOCK == slot[i] // BLOCK:
            j += 1
        page, b, o = slot[i] // P, slot[i] % P // BLOCK, slot[i] % BLOCK
        for h in range(values.shape[1]):
            x = new[i:j, h].astype(np.float64)
            bad = not np.isfinite(x).all()
            e = E_MIN if bad else exponent(np.abs(x).max(), codes)
            v = values[page, h, b]
            if o == 0:
                v[:] = 0
            elif np.isnan(scale[page, h, b]):
                bad = True
            else:
                f = int(math.frexp(scale[page, h, b])[1]) - 1
                e = max(e, f) if not bad else f
                if e > f:
                    v[:o] = nearest(v[:o] * 2.0 ** (f - e), codes)
            v[o:o + j - i] = 0 if bad else nearest(x * 2.0 ** -e, codes)
            scale[page, h, b] = math.nan if bad else 2.0 ** e
        i = j
    return values, scale


# ------------------------------------------------------------------------------------------------ attention
def attend(q, k, v, length, offs, table, P, *, scale, G, prefix=None, cap=0.0, slopes=None, tag=None, see=None, position=None, row_position=None,
           refused=()):
    """q [n, Hq, D]; k, v [n_slots, Hkv, D] values.  Returns out, lse, and for bounds of the error: sum_j w_j |v_j|, max |v| seen, max |s| seen."""
    n, Hq, D = q.shape
    out, lse, mean = np.zeros((n, Hq, D)), np.full((n, Hq), -math.inf), np.zeros((n, Hq, D))
    most_v, most_s = np.zeros((n, Hq)), np.zeros((n, Hq))
    n_pages = k.shape[0] // P
    for r in range(len(length)):
        lo, hi = offs[r], offs[r + 1]
        T = int(length[r])
        if lo == hi or r in refused:
            continue
        t = np.arange(T)
        page = table[r, t // P]
        there = (page >= 0) & (page < n_pages)
        slot = np.where(there, page, 0) * P + t % P
        for i in range(lo, hi):
            p = T - (hi - lo) + i - lo
            vis = t <= p
            if see is not None:
                vis &= np.array([(int(see[i]) >> int(tag[s] & 63)) & 1 for s in slot], bool)
            if prefix is not None:
                vis |= t < prefix[r]
            vis &= there
            if not vis.any():
                continue
            s_ = slot[vis]
            for h in range(Hq):
                kk, vv = k[s_, h // G], v[s_, h // G]
                z = kk @ q[i, h] * scale
                if cap:
                    z = cap * np.tanh(z / cap)
                if slopes is not None:
                    a, b = (t[vis], p) if row_position is None else (position[s_].astype(np.int64), int(row_position[i]))
                    z = z - float(slopes[h]) * np.abs(b - a)
                if np.isnan(z).any():
                    out[i, h], lse[i, h] = math.nan, math.nan
                    continue
                m = z.max()
                w = np.exp(z - m)
                lse[i, h] = m + math.log(w.sum())
                w /= w.sum()
                out[i, h], mean[i, h] = w @ vv, w @ np.abs(vv)
                most_v[i, h], most_s[i, h] = np.abs(vv).max(), np.abs(z).max()
    return out, lse, mean, most_v, most_s
