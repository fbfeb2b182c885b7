"""Softmax attention of one kv head in 64 bits, and how far a result of the paged cache's kernels may be from it."""
import math

import torch

from test_gpu_pages_precision import FLOOR, QUERY, WEIGHT


def attention(kind, q, K, V, seen, scale):
    """q [m, d], K [n, d], V [n, 128], seen [m]: the result [m, 128] and its error before it is rounded to the output's type (rows that
    see nothing: zeros and none).  The terms are those of test_gpu_pages_precision.check(): the scores' products added up in float32
    (a step, 2^-23, of the sum of magnitudes), q's rounding, three float32 roundings of exponents; the weights' rounding and its
    floor; 2^-21 for exp2 and the division; sums of n terms in steps of 16 at least."""
    q, K, V = q.double(), K.double(), V.double()
    n = K.shape[0]
    if n == 0:
        return torch.zeros(q.shape[0], V.shape[1], dtype=torch.float64, device=q.device), 0.0
    s = (q @ K.T) * scale
    hidden = torch.arange(n, device=s.device)[None, :] >= seen[:, None]
    nothing = (seen <= 0)[:, None]
    w = torch.softmax(s.masked_fill(hidden, -math.inf), dim=1).masked_fill(nothing, 0.0)
    want, share = w @ V, w @ V.abs()
    size = ((q.abs() @ K.abs().T) * scale * (K != 0).sum(dim=1)).masked_fill(hidden, 0.0).amax(dim=1)
    top_s = s.abs().masked_fill(hidden, 0.0).amax(dim=1)
    score = 2.0 ** -23 * size + QUERY[kind] * q.abs().amax(dim=1) * (K.abs().sum(dim=1).max() * scale) + 3 * 2.0 ** -24 * 2 * top_s
    rel = WEIGHT[kind] + 2 * score + 2.0 ** -21 + (n / 16) * 2.0 ** -23
    floor = FLOOR[kind] * n * w.amax(dim=1) * V.abs().max()
    return want, rel[:, None] * share + floor[:, None]


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def close(got, want, tol, what=""):
    """tol: before the rounding to got's type."""
    half = half_step(got.dtype)
    tol = half * want.abs() + (1 + half) * tol
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), (what, float((err - tol).max()), float(err.max()), float(want.abs().mean()))
