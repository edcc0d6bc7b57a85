"""float64 reference of the cached-history operators: rotary positions, appending to a
paged cache (bf16, or e4m3 with an exponent per page and head), reading pages back, and
attention over the cache.  Written from the definitions in include/cast.h with plain
loops; numpy only."""
from __future__ import annotations

import math

import numpy as np


# ---------------------------------------------------------------- rotation

def frequencies(dims, base=10000.0, scaling="none", factor=1.0, orig_len=0.0, beta_fast=32.0, beta_slow=1.0):
    turns, axis = [], []
    for a, d in enumerate(dims):
        for i in range(d // 2):
            t = base ** (-2.0 * i / d) / (2.0 * math.pi)
            if scaling == "linear":
                t /= factor
            elif scaling == "parts":
                g = min(1.0, max(0.0, (orig_len * t - beta_slow) / (beta_fast - beta_slow)))
                t = t * g + t / factor * (1.0 - g)
            turns.append(t)
            axis.append(a)
    return np.array(turns), np.array(axis)


def rope(x, pos, turns, axis=None, inter=False, amp=1.0, transpose=False):
    """x [n, H, dh] float64, pos [n, axes] integers."""
    y = np.array(x, dtype=np.float64)
    half = len(turns)
    pos = np.asarray(pos, dtype=np.int64).reshape(len(y), -1)
    for j in range(half):
        c0, c1 = (2 * j, 2 * j + 1) if inter else (j, j + half)
        rev = pos[:, 0 if axis is None else int(axis[j])].astype(np.float64) * float(turns[j])
        t = 2.0 * math.pi * (rev - np.round(rev))
        co, si = amp * np.cos(t)[:, None], amp * np.sin(t)[:, None] * (-1.0 if transpose else 1.0)
        a, b = np.array(x[..., c0], dtype=np.float64), np.array(x[..., c1], dtype=np.float64)
        y[..., c0], y[..., c1] = a * co - b * si, a * si + b * co
    return y


# ---------------------------------------------------------------- e4m3

def e4m3_values():
    """Value of each of the 256 codes (NaN for 0x7f and 0xff)."""
    v = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m * 2.0 ** -9 if e == 0 else (1.0 + m / 8.0) * 2.0 ** (e - 7)
        if c & 127 == 127:
            x = math.nan
        v[c] = -x if c & 128 else x
    return v


E4M3 = e4m3_values()
_POS = E4M3[:127]                    # 0 .. 448, ascending


def e4m3_code(x):
    """Nearest code of each finite |x| <= 448 (ties to the even code); others 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    hi = np.clip(np.searchsorted(_POS, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _POS[lo], _POS[hi] - a
    c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    c = np.where(a == _POS[hi], hi, c)
    c = np.where(np.signbit(x), c | 128, c)
    return np.where(np.isfinite(x), c, 0x7f).astype(np.uint8)


def need_exp(x):
    """Least e >= -117 with max |finite x| <= 448 * 2^e."""
    f = np.abs(x[np.isfinite(x)])
    top = float(f.max()) if f.size else 0.0
    e = -117
    while top > 448.0 * 2.0 ** e:
        e += 1
    return e


# ---------------------------------------------------------------- sequences

def tokens(cu, lens, n_seq):
    """(row, sequence, index in it) of every row that belongs to a sequence."""
    for b in range(n_seq):
        for r in range(cu[b], cu[b + 1]):
            yield r, b, lens[b] - (cu[b + 1] - r)


def append(cache, cu, lens, table, k, v):
    """Store rotated k and v [n, H, dh] into `cache` (dict of k, v [pages, page, H, dh] values
    or codes, and k_exp, v_exp for codes), in place."""
    pages, page, H, _ = cache["k"].shape
    limit = table.shape[1] * page
    for b in range(len(lens)):
        n = int(cu[b + 1] - cu[b])
        length = min(max(int(lens[b]), 0), limit)
        first = length - n
        groups = {}
        for r in range(n):
            t = first + r
            if t >= 0 and 0 <= table[b, t // page] < pages:
                groups.setdefault(t // page, []).append((int(cu[b]) + r, t % page))
        for g, rows in groups.items():
            at = table[b, g]
            rr, oo = [r for r, _ in rows], [o for _, o in rows]
            for name, x in (("k", k), ("v", v)):
                if cache.get(name + "_exp") is None:
                    cache[name][at, oo] = x[rr]
                    continue
                had = oo[0]
                for h in range(H):
                    e = need_exp(x[rr, h])
                    old = int(cache[name + "_exp"][at, h]) - 127
                    if had:
                        e = max(e, old)
                        if e > old:
                            cache[name][at, :had, h] = e4m3_code(E4M3[cache[name][at, :had, h]] * 2.0 ** (old - e))
                    cache[name + "_exp"][at, h] = e + 127
                    cache[name][at, oo, h] = e4m3_code(x[rr, h] * 2.0 ** -e)


def values(codes, exps):
    scale = np.where(exps == 255, math.nan, 2.0 ** (exps.astype(np.float64) - 127.0))
    return E4M3[codes] * scale[:, None, :, None]


# ---------------------------------------------------------------- attention

def attention(q, kv, vv, cu, lens, table, page, scale, causal=True, window=0, sinks=0):
    """q [n, Hq, dh]; kv, vv [pages, page, H, dh] values (float64).  Returns out (NaN rows where
    a row belongs to no sequence), lse, and sum_j p_j |v_j| of every output element."""
    n, Hq, dh = q.shape
    pages, _, H, _ = kv.shape
    g = Hq // H
    out = np.full((n, Hq, dh), math.nan)
    mag = np.full((n, Hq, dh), math.nan)
    lse = np.full((n, Hq), math.nan)
    for r, b, p in tokens(cu, lens, len(lens)):
        length = min(max(int(lens[b]), 0), table.shape[1] * page)
        p = length - (int(cu[b + 1]) - r)
        js = [j for j in range(length) if (not causal or j <= p) and (not window or j > p - window or j < sinks)
              and 0 <= table[b, j // page] < pages]
        if not js:
            out[r], mag[r], lse[r] = 0.0, 0.0, -math.inf
            continue
        at, row = table[b, np.array(js) // page], np.array(js) % page
        K, V = kv[at, row], vv[at, row]                     # [keys, H, dh]
        for h in range(Hq):
            s = scale * (K[:, h // g] @ q[r, h])
            m = s.max()
            e = np.exp(s - m)
            out[r, h] = (e / e.sum()) @ V[:, h // g]
            mag[r, h] = (e / e.sum()) @ np.abs(V[:, h // g])
            lse[r, h] = m + math.log(e.sum())
    return out, lse, mag
