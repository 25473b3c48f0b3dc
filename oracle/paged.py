"""fp64 definition of the operators over a paged cache: attention of new rows, the attention weight that cached rows
receive, which rows an eviction keeps.  Test infrastructure only."""
from __future__ import annotations

import math

import numpy as np

from .unigist_oracle import visible


def paged_rows(pool, pages, n):
    """pool [n_pages, Hkv, page, ...], pages: one sequence's table -> its rows 0 .. n-1 [Hkv, n, ...] and which of them lie
    in a page that is there (the others are zero)."""
    n_pages, Hkv, page = pool.shape[:3]
    out = np.zeros((Hkv, n) + pool.shape[3:], dtype=pool.dtype)
    there = np.zeros(n, dtype=bool)
    for j in range(n):
        if j // page < len(pages) and 0 <= pages[j // page] < n_pages:
            out[:, j] = pool[pages[j // page], :, j % page]
            there[j] = True
    return out, there


def paged_attn(q, k, v, table, kv_len, cu, r, W, sinks=0, units=False, weigh=0):
    """q [Hq, T, D]; k, v pools (float64, already code * scale); -> out [Hq, T, D], lse [Hq, T] (NaN where no sequence has the
    row), and per sequence the weight added to each of its rows, [Hkv, kv_len]."""
    Hq, T, D = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    out, lse, added = np.full((Hq, T, D), np.nan), np.full((Hq, T), np.nan), []
    for b, L in enumerate(int(x) for x in kv_len):
        t0, t1 = int(cu[b]), int(cu[b + 1])
        n = t1 - t0
        kb, there = paged_rows(k, table[b], L)
        vb, _ = paged_rows(v, table[b], L)
        add = np.zeros((Hkv, L))
        j = np.arange(L)
        for i in range(n):
            p = L - n + i
            vis = np.zeros(L, dtype=bool)
            if p >= 0:
                vis = visible(np.int64(p), j, r, W, sinks=sinks, units=units) & there
            for h in range(Hq):
                if not vis.any():
                    out[h, t0 + i], lse[h, t0 + i] = 0.0, -math.inf
                    continue
                s = kb[h // G][vis] @ q[h, t0 + i] / math.sqrt(D)
                m = s.max()
                e = np.exp(s - m)
                out[h, t0 + i] = e @ vb[h // G][vis] / e.sum()
                lse[h, t0 + i] = m + math.log(e.sum())
                if i >= n - weigh:
                    add[h // G, vis] += e / e.sum()
        added.append(add)
    return out, lse, added


def paged_select(weight, keep, sinks=0, recent=0):
    """weight [n] of one kv head of one sequence -> the rows kept, ascending: protected ones first (the first `sinks`, the
    last `recent`), then by weight, NaN least, ties to the lower row."""
    n = len(weight)
    key = [(0 if j < sinks or j >= n - recent else 1, 2 if math.isnan(w) else 1, 0.0 if math.isnan(w) else -float(w), j)
           for j, w in enumerate(weight)]
    return np.array(sorted(x[3] for x in sorted((0, 0, 0.0, j) if p == 0 else (p, a, w, j) for p, a, w, j in key)[:keep]), dtype=np.int64)
