"""Plain restatement, in Python lists and float64, of the paged cache's calls for shared pages and of differential attention."""
import numpy as np

import pages_ref as ref

pages_of = ref.pages_of


def fork(src, dst, length, kv, table, free, n_free, page):
    """Lists in, new lists out: kv, table, n_free, and (from page, to page, rows) of each page that is copied."""
    kv, table, copies = list(kv), [list(r) for r in table], []
    before, B = list(kv), len(kv)
    valid = [s >= 0 and s < B and 0 <= d < B for s, d in zip(src, dst)]
    sources = {s for s, ok in zip(src, valid) if ok}
    written = set()
    for i, (s, d) in enumerate(zip(src, dst)):
        if not valid[i] or d in sources or d in written:
            continue
        written.add(d)
        n = min(before[s], before[s] if length is None else length[i])
        whole, rest = divmod(n, page)
        if rest and n_free == 0:
            kv[d] = 0
            continue
        kv[d] = n
        table[d][:whole] = table[s][:whole]
        if rest:
            n_free -= 1
            table[d][whole] = free[n_free]
            copies.append((table[s][whole], free[n_free], rest))
    return kv, table, n_free, copies


def release(t, n_new, table, free, n_free, page):
    free = list(free)
    held = {p for b, n in enumerate(n_new) if n >= 0 for p in table[b][:pages_of(t[b], page)]}
    for b, n in enumerate(n_new):
        if n < 0:
            for p in table[b][:pages_of(t[b], page)]:
                if p not in held:
                    held.add(p)
                    free[n_free] = p
                    n_free += 1
    return free, n_free, [0 if n < 0 else x for x, n in zip(t, n_new)]


def compact(kv, table, free, n_pages, page):
    """table, free, n_free, new_id, and the pairs (from, to)."""
    live = {p for row, t in zip(table, kv) for p in row[:pages_of(t, page)]}
    n = len(live)
    moves = list(zip(sorted(p for p in live if p >= n), [p for p in range(n) if p not in live]))
    new = [p if p in live and p < n else -1 for p in range(n_pages)]
    for a, b in moves:
        new[a] = b
    table = [[new[p] if j < pages_of(t, page) else p for j, p in enumerate(row)] for row, t in zip(table, kv)]
    free = [n_pages - 1 - i if i < n_pages - n else x for i, x in enumerate(free)]
    return table, free, n_pages - n, new, moves


def attn_diff(q, q_start, kv_len, table, kc, ks, vc, vs, page, lam, gain=None, eps=0.0, scale=None):
    """q [n, HQ, 128] float64 -> out and the largest magnitude of the two maps' outputs, both of q's shape."""
    n, HQ, _ = q.shape
    H = kc.shape[1]
    G = HQ // H
    scale = 0.125 if not scale else scale
    out, size = np.full(q.shape, np.nan), np.zeros(q.shape)
    for b, L in enumerate(kv_len):
        K, V = ref.rows_of(kc, ks, table[b], L, page), ref.rows_of(vc, vs, table[b], L, page)
        m = q_start[b + 1] - q_start[b]
        for i in range(m):
            seen = L - m + i + 1
            for g in range(HQ):
                o = np.zeros(128)
                if seen > 0:
                    maps = []
                    for part in (slice(0, 64), slice(64, 128)):
                        s = K[g // G, :seen, part] @ q[q_start[b] + i, g, part] * scale
                        w = np.exp(s - s.max())
                        maps.append(w @ V[g // G, :seen] / w.sum())
                        size[q_start[b] + i, g] = np.maximum(size[q_start[b] + i, g], w @ np.abs(V[g // G, :seen]) / w.sum())
                    o = maps[0] - lam[g] * maps[1]
                if gain is not None:
                    r = np.sqrt((o * o).mean() + eps)
                    o = np.zeros(128) if r == 0 else o / r * gain
                out[q_start[b] + i, g] = o
    return out, size
