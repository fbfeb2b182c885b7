"""Plain restatement of the paged 8-bit cache in Python lists and float64, for the tests."""
import math

import numpy as np
import torch

E4M3_MAX = 448.0
D = 128


def e4m3_values() -> np.ndarray:
    """The 256 values: sign, 4 exponent bits (bias 7), 3 fraction bits, 0x7f / 0xff NaN, no infinities."""
    v = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        a = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[c] = math.nan if (c & 127) == 127 else (-a if c & 128 else a)
    return v


VALUES = e4m3_values()
_POS = VALUES[:127]                                  # ascending, 0 .. 448


def encode(x: np.ndarray) -> np.ndarray:
    """Codes of float64 values: nearest, ties to the even code, saturating; NaN to NaN."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(x), E4M3_MAX)
    a = np.where(np.isnan(a), 0.0, a)
    hi = np.searchsorted(_POS, a, side="left").clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _POS[lo], _POS[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = np.where(_POS[hi] == a, hi, code)
    code = np.where(np.isnan(x), 127, code)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_for(amax: float) -> float:
    s = 2.0 ** -126
    while amax / s > E4M3_MAX:
        s *= 2.0
    return s


def pages_of(n, page):
    return (n + page - 1) // page


def tables(t_len, n_new, table, free, n_free, n_tokens, page):
    """Lists in, new lists out: table, free, n_free, q_start, kv_len, slots."""
    table, free = [list(r) for r in table], list(free)
    W = len(table[0])
    for b, n in enumerate(n_new):
        if n < 0:
            for j in range(pages_of(t_len[b], page)):
                free[n_free] = table[b][j]
                n_free += 1
    start, kv, slots, stuck = [0], [], [-1] * n_tokens, False
    for b, n in enumerate(n_new):
        m = max(n, 0)
        first = start[-1]
        start.append(first + m)
        if n < 0:
            kv.append(0)
            continue
        t = t_len[b]
        have, want = pages_of(t, page), pages_of(t + m, page)
        if want > W or t + m > W * page or first + m > n_tokens:
            kv.append(t)
            continue
        if want > have and (stuck or want - have > n_free):
            stuck = True
            kv.append(t)
            continue
        for j in range(have, want):
            n_free -= 1
            table[b][j] = free[n_free]
        kv.append(t + m)
        for i in range(m):
            slots[first + i] = table[b][(t + i) // page] * page + (t + i) % page
    return table, free, n_free, start, kv, slots


def store(x, slots, codes, scales, page):
    """x [n, H, 128] float64, codes uint8 [n_pages, H, page, 128], scales float64 [n_pages, H]: new codes and scales."""
    codes, scales = codes.copy(), scales.copy()
    n, H, _ = x.shape
    runs = {}
    for i, s in enumerate(slots):
        if s >= 0:
            runs.setdefault(s // page, []).append((s % page, i))
    for p, rows in runs.items():
        r0 = rows[0][0]
        r, i = [a for a, _ in rows], [c for _, c in rows]
        for h in range(H):
            v = np.abs(x[i, h])
            amax = float(np.where(np.isfinite(v), v, 0.0).max())
            s = scale_for(amax)
            if r0 > 0 and scales[p, h] >= s:
                s = scales[p, h]
            elif r0 > 0:
                codes[p, h, :r0] = encode(VALUES[codes[p, h, :r0]] * scales[p, h] / s)
            scales[p, h] = s
            codes[p, h, r] = encode(x[i, h] / s)
    return codes, scales


def rows_of(codes, scales, table_row, n, page):
    """float64 rows [H, n, 128] of one sequence."""
    H = codes.shape[1]
    out = np.zeros((H, n, D))
    for j in range(pages_of(n, page)):
        p = table_row[j]
        k = min(page, n - j * page)
        out[:, j * page:j * page + k] = VALUES[codes[p, :, :k]] * scales[p][:, None, None]
    return out


def attn(q, q_start, kv_len, table, kc, ks, vc, vs, page, scale=None):
    """q [n, HQ, 128] float64 -> out, same shape (NaN rows where no sequence owns the token)."""
    n, HQ, _ = q.shape
    H = kc.shape[1]
    G = HQ // H
    scale = 1.0 / math.sqrt(D) if not scale else scale
    out = np.full(q.shape, np.nan)
    for b, L in enumerate(kv_len):
        K, V = rows_of(kc, ks, table[b], L, page), rows_of(vc, vs, table[b], L, page)
        m = q_start[b + 1] - q_start[b]
        for i in range(m):
            seen = L - m + i + 1
            for g in range(HQ):
                o = np.zeros(D)
                if seen > 0:
                    s = K[g // G, :seen] @ q[q_start[b] + i, g] * scale
                    w = np.exp(s - s.max())
                    o = w @ V[g // G, :seen] / w.sum()
                out[q_start[b] + i, g] = o
    return out


def spread(lens, page, n_pages, W, rng):
    """Block tables of scattered pages; entries behind a sequence's last page are out of range, so reading one would show."""
    perm = rng.permutation(n_pages)
    table = np.full((len(lens), W), 0x7fffffff, dtype=np.int64)
    at = 0
    for b, n in enumerate(lens):
        k = pages_of(n, page)
        table[b, :k] = perm[at:at + k]
        at += k
    return table


def random_cache(rng, n_pages, H, page, lens, table, pow2=True):
    """Codes and scales of written pages; every row that no sequence covers holds NaN codes."""
    codes = np.full((n_pages, H, page, D), 127, dtype=np.uint8)
    x = rng.standard_normal((n_pages, H, page, D))
    filled = encode(x * 100.0)
    for b, n in enumerate(lens):
        for j in range(pages_of(n, page)):
            k = min(page, n - j * page)
            codes[table[b, j], :, :k] = filled[table[b, j], :, :k]
    scales = 2.0 ** rng.integers(-9, -4, (n_pages, H)) if pow2 else rng.uniform(0.002, 0.02, (n_pages, H))
    return codes, scales.astype(np.float32).astype(np.float64)


def cuda8(codes):
    return torch.from_numpy(codes).cuda().view(torch.float8_e4m3fn)


def cuda32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.float32).cuda()


def ints(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32)).cuda()
