"""Attention over pages whose v_scales lie far apart, on the GPU against 64 bits.

What the calls state is that a softmax weight times its page's v_scale is held to a share of itself and of the row's largest such product: a
loud page whose tokens hardly count takes nothing from the others, in whatever order the pages come, and a page of zeros nothing at all."""
import math

import numpy as np
import pytest
import torch

import pages_ref as ref
from attn_bounds import close
from test_gpu_pages_precision import FLOOR, QUERY, WEIGHT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fk():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2507_20030_b200 import binding, build
    build.build()
    binding.load()
    return binding


def by_page(kind, q, K, codes, vs, seen, scale):
    """q [m, d], K [n, d], codes [n, 128], vs [n] (a token's v_scale): the result and its error before it is rounded.  As attn_bounds.attention(), but
    for the floor: of a weight times v_scale, in units of the row's largest, for every token that the row sees."""
    q, K = q.double(), K.double()
    n = K.shape[0]
    s = (q @ K.T) * scale
    hidden = torch.arange(n, device=s.device)[None, :] >= seen[:, None]
    w = torch.softmax(s.masked_fill(hidden, -math.inf), dim=1)
    V = codes * vs[:, None]
    want, share = w @ V, w @ V.abs()
    size = ((q.abs() @ K.abs().T) * scale * (K != 0).sum(dim=1)).masked_fill(hidden, 0.0).amax(dim=1)
    top_s = s.abs().masked_fill(hidden, 0.0).amax(dim=1)
    score = 2.0 ** -23 * size + QUERY[kind] * q.abs().amax(dim=1) * (K.abs().sum(dim=1).max() * scale) + 3 * 2.0 ** -24 * 2 * top_s
    rel = WEIGHT[kind] + 2 * score + 2.0 ** -21 + (n / 16) * 2.0 ** -23
    floor = FLOOR[kind] * (w * vs.abs()).amax(dim=1)[:, None] * ((~hidden).double() @ codes.abs())
    return want, rel[:, None] * share + floor


Q0 = 4.0                                                    # what every query has in channels 0 and 64, where only marked pages have keys


def mark(cache, pages, ratio, weight, scale):
    """The values of these pages 2^ratio times as large as the others', in the upper 64 channels alone; a token's weight times v_scale
    2^weight of the others' (and for pages of zeros, ratio None, its weight)."""
    kc, ks, vc, vs = cache
    nats = -(weight - (ratio or 0)) * math.log(2.0)
    for p in pages:
        kc[p] = 0
        kc[p, :, :, [0, 64]] = 254 if nats > 0 else 126      # 448 in magnitude
        ks[p] = np.float32(abs(nats) / (448.0 * Q0 * scale))
        if ratio is None:
            vc[p], vs[p] = 0, 2.0 ** -126
        else:
            vc[p, :, :, :64] = 0
            vs[p] = 2.0 ** (ratio - 7)


def loud(where, ratio, weight=-10):
    return lambda n, cache, row, scale: mark(cache, [row[int(w * (n - 1))] for w in where], ratio, weight, scale)


def zeros(where, weight):
    return lambda n, cache, row, scale: mark(cache, [row[int(w * (n - 1))] for w in where], None, weight, scale)


def signs(n, cache, row, scale):
    kc, ks, vc, vs = cache
    for i, p in enumerate(row[:n]):
        vs[p] *= (1.0, -1.0, 0.0, 1.0, 2.0 ** 12, -2.0 ** -12)[i % 6]


def no_values(n, cache, row, scale):                         # a scale of zero on every page but the last few
    cache[3][list(row[:max(1, n - 3)])] = 0.0


CASES = {
    "later26": loud([0.5], 26), "later40": loud([0.5], 40), "later55": loud([0.5], 55), "first26": loud([0.0], 26), "first40": loud([0.0], 40),
    "first55": loud([0.0], 55), "first75": loud([0.0], 75), "both50": loud([0.0, 0.3, 0.6, 0.95], 50), "heavy40": loud([0.4], 40, weight=8),
    "zeros_first": zeros([0.0], 3), "zeros_later": zeros([0.3, 0.7], 12), "zeros_and_loud": lambda *a: (zeros([0.2], 5)(*a), loud([0.6], 45)(*a)),
    "zeros_then_loud": lambda *a: (zeros([0.0], 5)(*a), loud([0.5], 45)(*a)), "tiny": lambda n, cache, row, scale: cache[3].fill(2.0 ** -117),
    "quiet": loud([0.1, 0.5, 0.9], -30, weight=-20), "signs": signs, "no_values": no_values,
}


def run(fk, call, dtype, page, H, G, lens, edit, new=None, shared=0, width=1, seed=0):
    """One call over a cache that edit(pages, cache, table row, scale) has changed for every sequence (for the first, where tokens are shared)."""
    rng = np.random.default_rng(sum(lens) + page + H + G + seed)
    B, counts = len(lens), new or [1] * len(lens)
    W = max(ref.pages_of(n, page) for n in lens) + width
    n_pages = sum(ref.pages_of(n, page) for n in lens) + 2
    table = ref.spread(lens, page, n_pages, W, rng)
    table[:, :shared // page] = table[0, :shared // page]
    (kc, ks), (vc, vs) = [ref.random_cache(rng, n_pages, H, page, lens, table) for _ in range(2)]
    kc[:, :, :, [0, 64]] = 0
    vs[:] = 2.0 ** -7
    scale = 0.125 if call == "attn_diff" else 1 / math.sqrt(128)
    cache = (kc, ks, vc, vs)
    for b in range(1 if shared else B):
        edit(ref.pages_of(shared or lens[b], page), cache, table[b], scale)
    pg = fk.Pages(n_kv_heads=H, n_q_heads=H * G, page_size=page, n_pages=n_pages, max_pages=W, max_batch=B,
                  kv_dtype=fk.BF16 if dtype == torch.bfloat16 else fk.F32)
    q = torch.from_numpy(rng.standard_normal((sum(counts), H * G, 128)))
    q[:, :, [0, 64]] = Q0 if call == "attn_diff" else Q0 / 2
    q = q.to(dtype).cuda()
    out = torch.full_like(q, 7.0)
    lam = torch.from_numpy(rng.uniform(0.2, 0.8, H * G)).float().cuda()
    start = np.concatenate([[0], np.cumsum(counts)])
    tensors = (ref.cuda8(kc), ref.cuda8(vc), ref.cuda32(ks), ref.cuda32(vs))
    q_start = None if new is None else ref.ints(start)
    if call == "attn":
        pg.attn(q, ref.ints(lens), ref.ints(table), *tensors, out, q_start=q_start)
    elif call == "attn_shared":
        pg.attn_shared(q, ref.ints(lens), ref.ints(table), ref.ints([0, B]), ref.ints([shared]), *tensors, out)
    else:
        pg.attn_diff(q, ref.ints(lens), ref.ints(table), *tensors, lam, out, q_start=q_start)
    many = new is not None or call == "attn_shared"
    kind = "f32" if dtype == torch.float32 else "wide" if many else "bf16"
    for b in range(B):
        n, rows = lens[b], slice(start[b], start[b + 1])
        K = torch.from_numpy(ref.rows_of(kc, ks, table[b], n, page)).cuda()
        codes = torch.from_numpy(ref.rows_of(vc, np.ones_like(vs), table[b], n, page)).cuda()
        token_vs = torch.from_numpy(np.repeat(vs[table[b][:ref.pages_of(n, page)]], page, axis=0)[:n]).cuda()
        seen = n - counts[b] + 1 + torch.arange(counts[b], device="cuda")
        for g in range(H * G):
            h = g // G
            if call == "attn_diff":
                (a1, e1), (a2, e2) = [by_page(kind, q[rows, g, part], K[h][:, part], codes[h], token_vs[:, h], seen, scale)
                                      for part in (slice(0, 64), slice(64, 128))]
                lm = float(lam[g])
                close(out[rows, g], a1 - lm * a2, e1 + abs(lm) * e2 + 3 * 2.0 ** -24 * (a1.abs() + abs(lm) * a2.abs()), (b, g))
            else:
                close(out[rows, g], *by_page(kind, q[rows, g], K[h], codes[h], token_vs[:, h], seen, scale), (b, g))
    assert pg.device_status() == 0
    pg.close()


# What the calls promise, in every form: scales within 2^40 of one another, and pages of zeros; the form with rows reaches further.
NEAR = {k: v for k, v in CASES.items() if not k[-2:].isdigit() or int(k[-2:]) <= 40} | {
    "later38": loud([0.5], 38), "first38": loud([0.0], 38), "both38": loud([0.0, 0.3, 0.6, 0.95], 38), "heavy38": loud([0.4], 38, weight=8),
    "zeros_and_loud": lambda *a: (zeros([0.2], 5)(*a), loud([0.6], 38)(*a)), "zeros_then_loud": lambda *a: (zeros([0.0], 5)(*a), loud([0.5], 38)(*a)),
    "zeros_then_very_loud": lambda *a: (zeros([0.0], 0)(*a), loud([0.5], 17 + 7, weight=17 + 7)(*a)),
    "quiet": loud([0.1, 0.5, 0.9], -38, weight=-20)}
EVERY = pytest.mark.parametrize("edit", list(CASES))
EVERY_NEAR = pytest.mark.parametrize("edit", list(NEAR))


@EVERY
@pytest.mark.parametrize("page,G,shared,rows", [(16, 8, 1600, 33), (64, 4, 2560, 20), (128, 2, 384, 64), (16, 1, 128, 40)])
def test_shared_columns_as_rows(fk, edit, page, G, shared, rows):
    run(fk, "attn_shared", torch.bfloat16, page, 1, G, [shared + 1 + i % 5 for i in range(rows)], CASES[edit], shared=shared, width=200000 // page * 16)


@EVERY
@pytest.mark.parametrize("page,G,lens,new", [(16, 4, [2000], [40]), (64, 2, [1500, 700], [20, 70]), (128, 1, [3000], [50])])
def test_differential_prompts_as_rows(fk, edit, page, G, lens, new):
    run(fk, "attn_diff", torch.bfloat16, page, 2, G, lens, CASES[edit], new, width=60000)


BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])


@EVERY_NEAR
@BOTH
@pytest.mark.parametrize("call", ["attn", "attn_diff"])
@pytest.mark.parametrize("page,G,lens", [(16, 4, [2000, 130]), (128, 1, [3000])])
def test_decode_steps(fk, edit, dtype, call, page, G, lens):
    run(fk, call, dtype, page, 2, G, lens, NEAR[edit])


@EVERY_NEAR
@BOTH
@pytest.mark.parametrize("page,G,shared,rows", [(16, 8, 1600, 3), (128, 2, 384, 2)])
def test_shared_columns_in_eights(fk, edit, dtype, page, G, shared, rows):
    run(fk, "attn_shared", dtype, page, 2, G, [shared + 1 + i % 5 for i in range(rows)], NEAR[edit], shared=shared)


@EVERY_NEAR
@BOTH
@pytest.mark.parametrize("call", ["attn", "attn_diff"])
@pytest.mark.parametrize("page,G,lens,new", [(16, 2, [900, 40, 300], [2, 1, 1])])
def test_new_tokens_in_eights(fk, edit, dtype, call, page, G, lens, new):
    run(fk, call, dtype, page, 2, G, lens, NEAR[edit], new)


@EVERY_NEAR
@pytest.mark.parametrize("page,G,lens,new", [(16, 8, [900, 1300], [40, 7]), (128, 1, [700, 140], [200, 1])])
def test_prompts_of_many_columns(fk, edit, page, G, lens, new):
    run(fk, "attn", torch.bfloat16, page, 2, G, lens, NEAR[edit], new)
