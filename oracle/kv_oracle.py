"""fp64 oracle of the decoding operators: rotary positions, the append to the paged cache of e4m3 codes and
attention over it, from their definitions in include/catq.h, one element, page and row after the other.
Test infrastructure only; shares no code with the library."""
from __future__ import annotations

import numpy as np

E4M3 = np.array([(-1.0 if c & 0x80 else 1.0) * (np.nan if (c & 0x7F) == 0x7F else
                 ((c & 7) / 8.0 * 2.0 ** -6 if (c >> 3 & 15) == 0 else (1 + (c & 7) / 8.0) * 2.0 ** ((c >> 3 & 15) - 7)))
                 for c in range(256)])
_POS = E4M3[:127]                         # 0 .. 448, increasing with the code
_MID = (_POS[:-1] + _POS[1:]) / 2


def e4m3_encode(x):
    """Codes of the nearest e4m3 numbers, ties to the even code, |x| <= 464 (what rounds to 448 at most)."""
    x = np.asarray(x, np.float64)
    a = np.abs(x)
    c = np.searchsorted(_MID, a, side="left")          # a tie stays below
    tie = (c < 126) & (a == _MID[np.minimum(c, 125)])
    c = np.where(tie & (c % 2 == 1), c + 1, c)
    return np.where(np.signbit(x), c | 0x80, c).astype(np.uint8)


def half_step(x):
    """Half the distance of the e4m3 numbers around x."""
    e = np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6)))
    return 2.0 ** (e - 4)


def scale_of(top):
    """The least power of two, 2^-60 or more, with top <= 448 scale; 0 for 0, NaN if not finite."""
    if not np.isfinite(top):
        return np.nan
    if top == 0:
        return 0.0
    k = -60
    while top > 448.0 * 2.0 ** k:
        k += 1
    return 2.0 ** k


def frequencies(rot, base, scaling="plain", factor=1.0, low=1.0, high=4.0, original=8192.0):
    """(radians a token of every pair, magnitude)."""
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        if scaling == "linear":
            f /= factor
        elif scaling == "bands":
            turns = original * f / (2 * np.pi)
            if turns <= low:
                f /= factor
            elif turns < high:
                w = (turns - low) / (high - low)
                f = (1 - w) * f / factor + w * f
        elif scaling == "yarn":
            def at(t):
                return rot * np.log(original / (t * 2 * np.pi)) / (2 * np.log(base))
            a, b = max(np.floor(at(high)), 0), min(np.ceil(at(low)), rot - 1)
            w = min(max((i - a) / max(b - a, 0.001), 0), 1)
            f = f / factor * w + f * (1 - w)
        out.append(f)
    return np.array(out), (0.1 * np.log(factor) + 1.0 if scaling == "yarn" else 1.0)


def rope(x, pos, freq, interleaved, magnitude=1.0, inverse=False):
    """x [T, heads, d] with the first 2 len(freq) elements of every head rotated to pos [T]."""
    y = np.array(x, np.float64)
    half = len(freq)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        th = (np.asarray(pos, np.float64) * freq[i])[:, None] * (-1.0 if inverse else 1.0)
        c, s = magnitude * np.cos(th), magnitude * np.sin(th)
        p, q = np.array(x[..., a], np.float64), np.array(x[..., b], np.float64)
        y[..., a], y[..., b] = p * c - q * s, p * s + q * c
    return y


def append(codes, scale, table, page, row_start, seq_len, x):
    """codes [n_pages, nkv, page, d] uint8 and scale [n_pages, nkv], changed in place, get x [T, nkv, d] (fp64).
    Returns the unrounded values / scale of every new element, NaN elsewhere (like codes)."""
    asked = np.full(codes.shape, np.nan)
    for b in range(len(seq_len)):
        n = row_start[b + 1] - row_start[b]
        first = seq_len[b] - n
        for pg in range(max(first, 0) // page, (max(seq_len[b], 1) - 1) // page + 1):
            lo, hi = max(first, 0, pg * page), min(seq_len[b], (pg + 1) * page)
            if hi <= lo:
                continue
            p, kept = table[b][pg], lo - pg * page
            rows = x[row_start[b] + lo - first:row_start[b] + hi - first]
            for h in range(codes.shape[1]):
                old = scale[p, h] if kept else 0.0
                want = scale_of(np.abs(rows[:, h]).max()) if np.isfinite(rows[:, h]).all() else np.nan
                now = np.nan if np.isnan(old) or np.isnan(want) else max(old, want)
                scale[p, h] = now
                if np.isnan(now):
                    codes[p, h, kept:kept + hi - lo] = 0
                    continue
                if now > old > 0:
                    codes[p, h, :kept] = e4m3_encode(E4M3[codes[p, h, :kept]] * (old / now))
                v = rows[:, h] / now if now > 0 else rows[:, h] * 0.0
                codes[p, h, kept:kept + hi - lo] = e4m3_encode(v)
                asked[p, h, kept:kept + hi - lo] = v
    return asked


def attention(k_codes, v_codes, k_scale, v_scale, table, page, row_start, seq_len, q, T, nh):
    """(O [T, nh, d], lse [T, nh], weighted |v|, floor): O NaN in rows outside every sequence.  weighted |v| is
    sum p |v|, floor max(p s_v) sum |code of v| over the row's tokens: what errors of the weights scale with."""
    nkv, d = k_codes.shape[1], k_codes.shape[3]
    O = np.full((T, nh, d), np.nan)
    lse = np.full((T, nh), np.nan)
    mag, low = np.zeros((T, nh, d)), np.zeros((T, nh, d))
    for b in range(len(seq_len)):
        r0, r1 = row_start[b], row_start[b + 1]
        pages = [table[b][i] for i in range(-(-seq_len[b] // page))]
        for h in range(nh):
            hk = h // (nh // nkv)
            if pages:
                kc = np.concatenate([E4M3[k_codes[p, hk]] for p in pages])[:seq_len[b]]
                vc = np.concatenate([E4M3[v_codes[p, hk]] for p in pages])[:seq_len[b]]
                ks = np.repeat([k_scale[p, hk] for p in pages], page)[:seq_len[b]].astype(np.float64)
                vs = np.repeat([v_scale[p, hk] for p in pages], page)[:seq_len[b]].astype(np.float64)
            for r in range(r0, r1):
                n = seq_len[b] - (r1 - r0) + (r - r0) + 1  # tokens the row sees
                if n <= 0:
                    O[r, h], lse[r, h] = 0.0, -np.inf
                    continue
                s = kc[:n] @ q[r, h].astype(np.float64) * ks[:n] / np.sqrt(d)
                m = s.max()
                p = np.exp(s - m)
                total = p.sum()
                O[r, h] = (p * vs[:n]) @ vc[:n] / total
                lse[r, h] = m + np.log(total)
                mag[r, h] = (p * vs[:n]) @ np.abs(vc[:n]) / total
                low[r, h] = (p * vs[:n]).max() * np.abs(vc[:n]).sum(axis=0) / total
    return O, lse, mag, low
