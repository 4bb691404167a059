"""CPU oracle of the paged-cache operators (numpy, fp64): rotary positions, append, attention of a chunk with the weights
that rows collect, eviction.  One loop per definition, no blocking, no code shared with the kernels."""
from __future__ import annotations

import math

import numpy as np


def rope_frequencies(rot, base=10000.0, scaling="none", factor=1.0, orig_len=0.0, low_turns=1.0, high_turns=32.0):
    out = []
    for i in range(rot // 2):
        f = float(base) ** (-2.0 * i / rot)
        if scaling == "linear":
            f /= factor
        elif scaling == "by_parts":
            s = min(1.0, max(0.0, (orig_len * f / (2 * math.pi) - low_turns) / (high_turns - low_turns)))
            f = f * s + f * (1 - s) / factor
        out.append(f)
    return np.array(out)


def rope(x, pos, freq, interleaved, sign=1.0, out_scale=1.0):
    """x [.., n, D] turned by the angles sign * pos [.., n] * freq; the elements beyond 2 len(freq) are copied."""
    x = np.asarray(x, dtype=np.float64)
    out = x.copy()
    a = sign * np.asarray(pos, dtype=np.float64)[..., None] * freq
    r = 2 * len(freq)
    for i in range(len(freq)):
        u, v = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
        c, s = np.cos(a[..., i]), np.sin(a[..., i])
        out[..., u] = (x[..., u] * c - x[..., v] * s) * out_scale
        out[..., v] = (x[..., u] * s + x[..., v] * c) * out_scale
    return out


class Pool:
    """Pages K, V [n_pages, page_rows, D] and a table [B, Hkv, pages_cap]."""

    def __init__(self, K, V, table):
        self.K, self.V, self.table = (np.array(x) for x in (K, V, table))
        self.K, self.V = self.K.astype(np.float64), self.V.astype(np.float64)
        self.page_rows = self.K.shape[1]
        self.cap = self.table.shape[2] * self.page_rows

    def at(self, b, g, j):
        """(page, row in the page) of row j, or None."""
        page = self.table[b, g, j // self.page_rows]
        return (page, j % self.page_rows) if 0 <= page < len(self.K) else None


def append(pool, K, V, pos, new_cnt, row_cnt, row_pos, acc, freq=None, interleaved=False):
    """Stores the rows (in place in pool, row_pos, acc); returns row_end."""
    B, Hkv, n, _ = K.shape
    row_end = np.zeros((B, Hkv), dtype=np.int32)
    for b in range(B):
        cnt = min(max(int(new_cnt[b]), 0), n)
        for g in range(Hkv):
            have = min(max(int(row_cnt[b, g]), 0), pool.cap)
            row_end[b, g] = min(pool.cap, have + cnt)
            for t in range(cnt):
                j = have + t
                if j >= pool.cap:
                    break
                row_pos[b, g, j] = pos[b] + t
                if acc is not None:
                    acc[b, g, j] = 0
                at = pool.at(b, g, j)
                if at:
                    k = K[b, g, t]
                    pool.K[at] = k if freq is None else rope(k[None], [pos[b] + t], freq, interleaved)[0]
                    pool.V[at] = V[b, g, t]
    return row_end


def attend(Q, pool, row_end, new_cnt, causal, scale):
    """O, lse, weights [B,Hkv,cap] of the chunk, and per output the sums that error bounds are made of: pv = sum p |v| (like
    O), qk = the largest sum |q k| scale among the rows a query row sees (like lse)."""
    B, Hq, n, D = Q.shape
    Hkv = pool.table.shape[1]
    G = Hq // Hkv
    Q = np.asarray(Q, dtype=np.float64)
    O, pv = np.zeros(Q.shape), np.zeros(Q.shape)
    lse, qk = np.full((B, Hq, n), -np.inf), np.zeros((B, Hq, n))
    weights = np.zeros((B, Hkv, pool.cap))
    for b in range(B):
        cnt = min(max(int(new_cnt[b]), 0), n)
        for g in range(Hkv):
            end = min(max(int(row_end[b, g]), 0), pool.cap)
            rows = [j for j in range(end) if pool.at(b, g, j)]
            if not rows:
                continue
            where = [pool.at(b, g, j) for j in rows]
            k, v = np.array([pool.K[w] for w in where]), np.array([pool.V[w] for w in where])
            rows = np.array(rows)
            for i in range(g * G, (g + 1) * G):
                for t in range(cnt):
                    seen = rows < (end - cnt + t + 1 if causal else end)
                    if not seen.any():
                        continue
                    q, ks, vs = Q[b, i, t], k[seen], v[seen]
                    z = ks @ q * scale
                    top = z.max()
                    e = np.exp(z - top)
                    p = e / e.sum()
                    O[b, i, t], pv[b, i, t] = p @ vs, p @ np.abs(vs)
                    lse[b, i, t] = top + math.log(e.sum())
                    qk[b, i, t] = (np.abs(ks) @ np.abs(q)).max() * scale
                    weights[b, g, rows[seen]] += p
    return O, lse, weights, pv, qk


def evict(pool, budget, n_sink, n_recent, seq_len, row_end, row_pos, acc):
    """Moves rows in the pool; returns row_cnt, row_pos, acc (the last two: rows below row_cnt are what counts)."""
    B, Hkv, _ = pool.table.shape
    row_pos, acc, row_cnt = row_pos.copy(), acc.copy(), np.zeros((B, Hkv), dtype=np.int32)
    for b in range(B):
        for g in range(Hkv):
            end = min(max(int(row_end[b, g]), 0), pool.cap)
            keep = min(end, budget)
            row_cnt[b, g] = keep

            def rank(j):
                if row_pos[b, g, j] < n_sink or row_pos[b, g, j] >= int(seq_len[b]) - n_recent:
                    return (0, 0.0, j)
                w = acc[b, g, j]
                return (1, math.inf if math.isnan(w) else -float(w), j)
            stay = set(sorted(range(end), key=rank)[:keep])
            holes = [j for j in range(keep) if j not in stay]
            movers = [j for j in range(keep, end) if j in stay]
            for to, frm in zip(holes, movers):
                row_pos[b, g, to], acc[b, g, to] = row_pos[b, g, frm], acc[b, g, frm]
                src, dst = pool.at(b, g, frm), pool.at(b, g, to)
                if src and dst:
                    pool.K[dst], pool.V[dst] = pool.K[src], pool.V[src]
    return row_cnt, row_pos, acc
