"""TEST INFRASTRUCTURE -- keys and values in pages, in plain Python and fp64 numpy.

The page lists (table rows, lengths, owners) are updated one sequence and one page at
a time, as their definition reads; the attention gathers a sequence's tokens and takes
the softmax row by row.  Nothing here is shared with the library.
"""
from __future__ import annotations

import numpy as np


def _copies(table, lens, ref):
    return [list(map(int, r)) for r in table], list(map(int, lens)), list(map(int, ref))


def reserve(table, lens, ref, n_new, page):
    """Pages for n_new[b] more tokens; returns (table, lens, ref, missing)."""
    table, lens, ref = _copies(table, lens, ref)
    new = [max(int(n), 0) for n in n_new]
    have = [-(-max(n, 0) // page) for n in lens]
    want = [-(-(max(n, 0) + m) // page) for n, m in zip(lens, new)]
    free = [p for p, r in enumerate(ref) if r == 0]
    need = sum(w - h for h, w in zip(have, want))
    lack = max(need - len(free), 0) + sum(max(w - len(table[0]), 0) for w in want)
    if lack:
        return table, lens, ref, lack
    for b in range(len(lens)):
        for j in range(have[b], want[b]):
            p = free.pop(0)
            table[b][j], ref[p] = p, 1
        lens[b] = max(lens[b], 0) + new[b]
    return table, lens, ref, 0


def fork(table, lens, ref, src, dst, page):
    """dst[i] becomes a copy of src[i]; returns (table, lens, ref, copy_src, copy_dst,
    missing)."""
    table, lens, ref = _copies(table, lens, ref)
    B, n = len(lens), len(src)
    pairs, seen = [], set()
    for i, (a, b) in enumerate(zip(map(int, src), map(int, dst))):
        if not (0 <= a < B and 0 <= b < B) or b in seen or not (
                0 < lens[a] <= len(table[0]) * page and lens[b] <= 0):
            continue
        seen.add(b)
        pairs.append((i, a, b))
    free = [p for p, r in enumerate(ref) if r == 0]
    lack = max(sum(lens[a] % page > 0 for _, a, _ in pairs) - len(free), 0)
    copy_src, copy_dst = [-1] * n, [-1] * n
    if lack:
        return table, lens, ref, copy_src, copy_dst, lack
    for i, a, b in pairs:
        full, row = lens[a] // page, [-1] * len(table[0])
        for j in range(full):
            row[j] = table[a][j]
            if 0 <= row[j] < len(ref):
                ref[row[j]] += 1
        if lens[a] % page:
            row[full] = free.pop(0)
            ref[row[full]] = 1
            copy_src[i], copy_dst[i] = table[a][full], row[full]
        table[b] = row
    for _, a, b in pairs:
        lens[b] = lens[a]
    return table, lens, ref, copy_src, copy_dst, 0


def free(table, lens, ref, seqs, page):
    """The sequences of seqs give up their pages; returns (table, lens, ref)."""
    table, lens, ref = _copies(table, lens, ref)
    for b in sorted({int(b) for b in seqs if 0 <= b < len(lens)}):
        for j in range(min(-(-max(lens[b], 0) // page), len(table[b]))):
            if 0 <= table[b][j] < len(ref):
                ref[table[b][j]] -= 1
        table[b] = [-1] * len(table[b])
        lens[b] = 0
    return table, lens, ref


def compact(table, ref):
    """The pages in use become the first ones; returns (table, ref, move_src, move_dst,
    counts), the moves filled up with -1 to len(ref) // 2."""
    table, _, ref = _copies(table, [], ref)
    used = [p for p, r in enumerate(ref) if r > 0]
    src = [p for p in used if p >= len(used)]
    dst = [p for p in range(len(used)) if ref[p] <= 0]
    to = dict(zip(src, dst))
    table = [[to.get(p, p) for p in row] for row in table]
    for a, b in to.items():
        ref[b], ref[a] = ref[a], 0
    pad = [-1] * (len(ref) // 2 - len(src))
    return table, ref, src + pad, dst + pad, [len(used), len(src)]


def paged_attention(q, k_pages, v_pages, table, lens, scale, q_len=None, causal=False):
    """(o, lse, size) in fp64: size[b,h,s,:] is the softmax mean of |v|, the scale of
    what rounding the weights can change.  Rows from q_len[b] on are NaN."""
    B, Hq, S, d = q.shape
    n_pages, Hkv, page, _ = k_pages.shape
    o = np.full((B, Hq, S, d), np.nan)
    size = np.full((B, Hq, S, d), np.nan)
    lse = np.full((B, Hq, S), np.nan)
    for b in range(B):
        new = S if q_len is None else int(q_len[b])
        held = min(max(int(lens[b]), 0), len(table[b]) * page)  # later tokens have no page
        at = [t for t in range(held) if 0 <= table[b][t // page] < n_pages]
        pos = np.array(at, dtype=np.int64)
        ids = np.array([table[b][t // page] for t in at], dtype=np.int64)
        for h in range(Hq):
            k = k_pages[ids, h * Hkv // Hq, pos % page].astype(np.float64)
            v = v_pages[ids, h * Hkv // Hq, pos % page].astype(np.float64)
            for s in range(new):
                x = scale * (k @ q[b, h, s].astype(np.float64))
                see = pos <= int(lens[b]) - new + s if causal else np.ones(len(at), bool)
                x = x[see]
                m = x.max() if len(x) else -np.inf
                if m == -np.inf:
                    o[b, h, s], lse[b, h, s], size[b, h, s] = 0.0, -np.inf, 0.0
                    continue
                w = np.exp(x - m)
                lse[b, h, s] = m + np.log(w.sum())
                o[b, h, s] = w @ v[see] / w.sum()
                size[b, h, s] = w @ np.abs(v[see]) / w.sum()
    return o, lse, size
