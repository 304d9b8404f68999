"""Paged caches in float64 NumPy: block tables from request lengths, rows to slots, attention over pages.

Written from the definitions in include/rkv.h; parity unpinned by the paper, which has no paged cache.
"""
import math

import numpy as np


def resize(table, lens, ring, cursor, new_lens, page_size, max_new):
    """The state after a resize, as lists: table, lens, ring, cursor, slots, cu_new, status."""
    table, ring = [list(r) for r in table], list(ring)
    head, count = cursor
    n_pages, width = len(ring), len(table[0]) if table else 0
    have = [-(-a // page_size) for a in lens]
    want = [-(-a // page_size) for a in new_lens]
    taken = sum(max(0, w - h) for h, w in zip(have, want))
    given = sum(max(0, h - w) for h, w in zip(have, want))
    added = sum(max(0, b - a) for a, b in zip(lens, new_lens))
    bad = any(x < 0 or x > width * page_size for x in list(lens) + list(new_lens)) or added > max_new
    bad = bad or not (0 <= head < n_pages and 0 <= count <= n_pages)
    bad = bad or (taken <= count and count - taken + given > n_pages)
    status = 2 if bad else 1 if taken > count else 0
    if status:
        return {"table": table, "lens": list(lens), "ring": ring, "cursor": [head, count], "slots": [-1] * max_new,
                "cu_new": [0] * (len(lens) + 1), "status": status}
    at = 0
    for s, (h, w) in enumerate(zip(have, want)):
        for j in range(h, w):
            table[s][j] = ring[(head + at) % n_pages]
            at += 1
    back = [table[s][j] for s, (h, w) in enumerate(zip(have, want)) for j in range(w, h)]
    for i, page in enumerate(back):
        ring[(head + count + i) % n_pages] = page
    slots, cu = [], [0]
    for s, (a, b) in enumerate(zip(lens, new_lens)):
        slots += [table[s][i // page_size] * page_size + i % page_size for i in range(a, b)]
        cu.append(len(slots))
    return {"table": table, "lens": list(new_lens), "ring": ring, "cursor": [(head + taken) % n_pages, count - taken + given],
            "slots": slots + [-1] * (max_new - len(slots)), "cu_new": cu, "status": 0}


def attend(k_pages, v_pages, q, table, lens, cu_q=None, *, scale=None, causal=True, window=0, softcap=0.0, slopes=None,
           prefix_lens=None, first_keys=None):
    """(out, lse, weight, reach) of every row and head: `weight` is sum_j p_j |v_j| (what a relative error of the
    probabilities moves an output by, at most), `reach` the largest scale sum_i |q_i k_ji| of the row's slots (what a relative
    error of the products moves a score by).  Rows of no sequence: nan."""
    n_pages, hkv, page_size, d = k_pages.shape
    T, hq, _ = q.shape
    g = hq // hkv
    scale = d ** -0.5 if scale is None else scale
    cu_q = list(range(len(lens) + 1)) if cu_q is None else [int(c) for c in cu_q]
    out, weight = np.full((T, hq, d), np.nan), np.full((T, hq, d), np.nan)
    lse, reach = np.full((T, hq), np.nan), np.zeros((T, hq))
    for s, n in enumerate(int(x) for x in lens):
        m = cu_q[s + 1] - cu_q[s]
        slot = [int(table[s][j // page_size]) for j in range(n)]
        for i in range(m):
            t, p = cu_q[s] + i, n - m + i
            hi = n if not causal else min(n, max(p + 1, int(prefix_lens[s]) if prefix_lens is not None else 0))
            lo = max(0, p - window + 1 if window else 0, int(first_keys[t]) if first_keys is not None else 0)
            j = np.arange(lo, max(lo, hi))
            page = np.array([slot[x] for x in j], dtype=np.int64)
            ok = (page >= 0) & (page < n_pages)
            page = np.where(ok, page, 0)
            for h in range(hkv):
                k = np.where(ok[:, None], k_pages[page, h, j % page_size].astype(np.float64), 0.0)
                v = np.where(ok[:, None], v_pages[page, h, j % page_size].astype(np.float64), 0.0)
                for e in range(h * g, (h + 1) * g):
                    if not len(j):
                        out[t, e], weight[t, e], lse[t, e] = 0.0, 0.0, -math.inf
                        continue
                    x = k @ q[t, e].astype(np.float64) * scale
                    reach[t, e] = np.abs(scale) * (np.abs(k) @ np.abs(q[t, e]).astype(np.float64)).max()
                    if softcap:
                        x = softcap * np.tanh(x / softcap)
                    if slopes is not None:
                        x = x - float(slopes[e]) * np.abs(p - j)
                    top = x.max()
                    w = np.exp(x - top)
                    total = w.sum()
                    out[t, e], weight[t, e], lse[t, e] = (w / total) @ v, (w / total) @ np.abs(v), top + math.log(total)
    return out, lse, weight, reach
