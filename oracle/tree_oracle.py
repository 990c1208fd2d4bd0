"""fp64 oracle of the calls around a tree of drafted tokens: what its rows see, attention over the cache, drawing a token,
the accepted branch and its compaction, from their definitions in include/catq.h, one row, token and page after the other.
Test infrastructure only; shares no code with the library."""
from __future__ import annotations

import math

import numpy as np

from oracle.kv_oracle import E4M3, e4m3_encode, scale_of


def ancestors(parent):
    """Every row's set of itself and its ancestors, for one tree (parents at or behind their row count as none)."""
    out = []
    for i, p in enumerate(parent):
        out.append({i} | (out[p] if 0 <= p < i else set()))
    return out


def masks(parent, row_start, seq_len, words):
    """(seen [T, words] uint32, positions [T]); rows outside every sequence 0 and -1."""
    T = len(parent)
    seen, pos = np.zeros((T, words), np.uint32), np.full(T, -1, np.int64)
    for b in range(len(seq_len)):
        r0, r1 = row_start[b], row_start[b + 1]
        for i, s in enumerate(ancestors(parent[r0:r1])):
            for j in s:
                seen[r0 + i, j // 32] |= np.uint32(1 << (j % 32))
            pos[r0 + i] = seq_len[b] - (r1 - r0) + len(s) - 1
    return seen, pos


def attention(k_codes, v_codes, k_scale, v_scale, table, page, row_start, seq_len, seen, q, nh):
    """As kv_oracle.attention, the rows' sight of their sequence's new tokens by bits."""
    nkv, d, T = k_codes.shape[1], k_codes.shape[3], q.shape[0]
    O, lse = np.full((T, nh, d), np.nan), np.full((T, nh), np.nan)
    mag, low = np.zeros((T, nh, d)), np.zeros((T, nh, d))
    for b in range(len(seq_len)):
        r0, r1, n = int(row_start[b]), int(row_start[b + 1]), int(seq_len[b])
        first = n - (r1 - r0)
        where = [(table[b][t // page], t % page) for t in range(n)]
        for h in range(nh):
            hk = h // (nh // nkv)
            for r in range(r0, r1):
                sees = [t for t in range(n)
                        if t < first or int(seen[r, (t - first) // 32]) >> ((t - first) % 32) & 1]
                if not sees:
                    O[r, h], lse[r, h] = 0.0, -np.inf
                    continue
                p_, at = np.array([where[t] for t in sees]).T
                ks, vs = k_scale[p_, hk].astype(np.float64), v_scale[p_, hk].astype(np.float64)
                kc, vc = E4M3[k_codes[p_, hk, at]], E4M3[v_codes[p_, hk, at]]
                s = kc @ q[r, h].astype(np.float64) * ks / np.sqrt(d)
                m = s.max()
                w = np.exp(s - m)
                total = w.sum()
                O[r, h] = (w * vs) @ vc / total
                lse[r, h] = m + np.log(total)
                mag[r, h] = (w * vs) @ np.abs(vc) / total
                low[r, h] = (w * vs).max() * np.abs(vc).sum(axis=0) / total
    return O, lse, mag, low


def sample(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, ln of its probability) of one row of logits, in whole numbers."""
    x = np.asarray(x, np.float64)
    if np.isnan(x).any() or x.max() in (np.inf, -np.inf) or not temperature >= 0:
        return -1, math.nan
    order = sorted(range(len(x)), key=lambda i: (-x[i], i))
    if temperature == 0:
        return order[0], 0.0
    temperature = min(max(float(temperature), 2.0 ** -60), 2.0 ** 60)
    w = [int(np.rint(2.0 ** 40 * np.exp((x[i] - x[order[0]]) / temperature))) for i in order]
    kept = len(w) if top_k <= 0 else min(int(top_k), len(w))
    whole = sum(w[:kept])
    if top_p < 1:
        need, run = min(max(math.ceil(float(top_p) * float(whole)), 1), whole), 0
        for i, v in enumerate(w):
            run += v
            if run >= need:
                kept = min(kept, i + 1)
                break
    least = max(1, math.ceil(2.0 ** 40 * min(float(min_p), 1.0))) if min_p > 0 else 1
    kept = min(kept, sum(v >= least for v in w))
    total = sum(w[:kept])
    at = math.floor(float(u) * float(total)) if u > 0 else 0
    at, run = min(at, total - 1), 0
    for i, v in zip(order, w):
        run += v
        if run > at:
            return i, math.log(v / total)


def accept(drafted, sampled, parent, row_start, seq_len):
    """(path [T], kept, next, new length [B])."""
    path = np.full(len(parent), -1, np.int64)
    kept, nxt, new_len = [], [], []
    for b in range(len(seq_len)):
        r0, n = row_start[b], row_start[b + 1] - row_start[b]
        way = [0] if n else []
        while way:
            token = sampled[r0 + way[-1]]
            fits = [i for i in range(way[-1] + 1, n) if parent[r0 + i] == way[-1] and drafted[r0 + i] == token >= 0]
            if not fits:
                break
            way.append(fits[0])
        path[r0:r0 + len(way)] = way
        kept.append(len(way))
        nxt.append(sampled[r0 + way[-1]] if way else -1)
        new_len.append(seq_len[b] - n + len(way))
    return path, np.array(kept), np.array(nxt), np.array(new_len)


def compact(codes, scale, table, page, row_start, seq_len, path, kept):
    """codes [n_pages, nkv, page, d] uint8 and scale [n_pages, nkv] (keys or values of one cache), changed in place."""
    old_codes, old_scale = codes.copy(), scale.copy()
    for b in range(len(seq_len)):
        r0, first = row_start[b], seq_len[b] - (row_start[b + 1] - row_start[b])
        moves = [(first + j, first + path[r0 + j]) for j in range(kept[b]) if path[r0 + j] != j and first + j >= 0]
        for pg in sorted({dst // page for dst, _ in moves}):
            p = table[b][pg]
            mine = [m for m in moves if m[0] // page == pg]
            for h in range(codes.shape[1]):
                came = [E4M3[old_codes[table[b][s // page], h, s % page]] * old_scale[table[b][s // page], h]
                        for _, s in mine]
                far = [v for v, (_, s) in zip(came, mine) if s // page != pg]
                want = 0.0
                if far:
                    want = scale_of(np.abs(far).max()) if np.isfinite(far).all() else np.nan
                now = np.nan if np.isnan(want) or np.isnan(old_scale[p, h]) else max(old_scale[p, h], want)
                scale[p, h] = now
                if np.isnan(now):
                    for dst, s in mine:  # inside a page a copy, finite codes else
                        codes[p, h, dst % page] = old_codes[p, h, s % page] if s // page == pg else 0
                    continue
                if now > old_scale[p, h] > 0:
                    codes[p, h] = e4m3_encode(E4M3[old_codes[p, h]] * (old_scale[p, h] / now))
                for (dst, s), v in zip(mine, came):
                    codes[p, h, dst % page] = e4m3_encode(v / now) if now > 0 else old_codes[table[b][s // page], h, s % page]
