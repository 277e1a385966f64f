"""fp64 oracle of the chunk attention over paged caches: every new token of a question attends the sink, the question's
selected groups and its own keys up to itself (Sec. 2.2, for several tokens at once).  Written from that sentence, row by
row of keys; it shares nothing with the product."""
from __future__ import annotations

import numpy as np


def own_rows(table_row, n: int, page_tokens: int, n_pages: int):
    """-> (cache rows of own keys 0 .. n-1, their index j) without those on pages that are not there."""
    j = np.arange(n)
    page = np.asarray(table_row, np.int64)[j // page_tokens] if n else np.zeros(0, np.int64)
    there = (page >= 0) & (page < n_pages)
    return (page * page_tokens + j % page_tokens)[there], j[there]


def chunk_attn(q, k_pool, v_pool, k_pages, v_pages, table, self_len, sink_len, demo_offsets, group_demo_offsets, cu_qlens,
               sel_ptr, sel_idx, scale):
    """-> dict(o [T, Hq, D], lse [Hq, T], weight [T, Hq, D] = sum p |v|, reach [T, Hq] = largest scale * sum |q k| of a visible
    key, keys [T]).  A row without keys: o = 0, lse = -inf.  page axes: k_pages [P, page tokens, Hkv, D]."""
    T, hq, d = q.shape
    hkv = k_pool.shape[1]
    r = hq // hkv
    bounds = np.asarray(demo_offsets)[np.asarray(group_demo_offsets)]
    n_pages, page_tokens = k_pages.shape[:2]
    out = dict(o=np.zeros((T, hq, d)), lse=np.full((hq, T), -np.inf), weight=np.zeros((T, hq, d)), reach=np.zeros((T, hq)),
               keys=np.zeros(T, np.int64))
    kp, vp = (x.reshape(n_pages * page_tokens, hkv, d) for x in (k_pages, v_pages))
    for u in range(len(cu_qlens) - 1):
        rows = [np.arange(sink_len)]
        for g in sel_idx[sel_ptr[u]:sel_ptr[u + 1]]:
            rows.append(np.arange(bounds[g], bounds[g + 1]))
        rows = np.concatenate(rows).astype(np.int64)
        n = min(max(int(self_len[u]), 0), table.shape[1] * page_tokens)
        at, j = own_rows(table[u], n, page_tokens, n_pages)
        k = np.concatenate([k_pool[rows], kp[at]])
        v = np.concatenate([v_pool[rows], vp[at]])
        index = np.concatenate([np.full(len(rows), -1), j])
        lo, hi = int(cu_qlens[u]), int(cu_qlens[u + 1])
        for t in range(lo, hi):
            pos = n - (hi - lo) + (t - lo)
            seen = (index < 0) | (index <= pos)
            out["keys"][t] = int(seen.sum())
            if not seen.any():
                continue
            for h in range(hq):
                kk, vv = k[seen, h // r], v[seen, h // r]
                s = scale * (kk @ q[t, h])
                top = s.max()
                p = np.exp(s - top)
                z = p.sum()
                out["o"][t, h] = (p @ vv) / z
                out["weight"][t, h] = (p @ np.abs(vv)) / z
                out["lse"][h, t] = top + np.log(z)
                out["reach"][t, h] = scale * (np.abs(kk) @ np.abs(q[t, h])).max()
    return out
