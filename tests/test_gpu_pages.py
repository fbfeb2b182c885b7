"""The paged 8-bit cache on the GPU against the plain reference: tables, store, attention, load, and a run of them."""
import math

import numpy as np
import pytest
import torch

import pages_ref as ref
from helpers import Guarded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fk():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2507_20030_b200 import binding, build
    build.build()
    binding.load()
    return binding


def make(fk, H=2, G=1, page=16, n_pages=40, W=8, B=8, dtype=torch.bfloat16):
    return fk.Pages(n_kv_heads=H, n_q_heads=H * G, page_size=page, n_pages=n_pages, max_pages=W, max_batch=B,
                    kv_dtype=fk.BF16 if dtype == torch.bfloat16 else fk.F32)


# ------------------------------------------------------------------------------------------------ tables

def _requests(rng, B, page, W, n_pages, tokens_most):
    t = rng.integers(0, max(1, W * page // 2), B)
    n = np.minimum(rng.integers(-1, max(2, tokens_most), B), W * page)
    held = [ref.pages_of(int(x), page) for x in t]
    perm = rng.permutation(n_pages)
    table = np.full((B, W), -7, dtype=np.int64)
    at = 0
    for b in range(B):
        while at + held[b] > n_pages:
            t[b] = max(0, t[b] // 2)
            held[b] = ref.pages_of(int(t[b]), page)
        table[b, :held[b]] = perm[at:at + held[b]]
        at += held[b]
    free = np.full(n_pages, -9, dtype=np.int64)
    free[:n_pages - at] = perm[at:]
    return t, n, table, free, n_pages - at


@pytest.mark.parametrize("B,page,W,n_pages,most,extra", [
    (1, 16, 4, 6, 2, 0),            # one request
    (16, 64, 40, 900, 2, 0),        # decode
    (7, 16, 20, 60, 50, 3),         # pages run out; padding behind the last token
    (7, 32, 3, 60, 200, 0),         # rows of the table run out
    (300, 16, 9, 2000, 60, 5),      # more tokens than one CTA places
    (1500, 16, 5, 6000, 4, 0),      # more requests than threads
    (40, 128, 70, 2000, 3000, -100),  # fewer token rows than tokens
])
def test_tables(fk, B, page, W, n_pages, most, extra):
    rng = np.random.default_rng(B * page + W)
    for trial in range(3):
        t, n, table, free, n_free = _requests(rng, B, page, W, n_pages, most)
        tokens = max(0, int(np.maximum(n, 0).sum()) + extra)
        want = ref.tables(t.tolist(), n.tolist(), table.tolist(), free.tolist(), n_free, tokens, page)
        pg = make(fk, page=page, n_pages=n_pages, W=W, B=B)
        slots, q_start = Guarded((tokens,), torch.int32, -5), Guarded((B + 1,), torch.int32, -5)
        for in_place in (False, True):
            d_t, d_n, d_table, d_free, d_nf = ref.ints(t), ref.ints(n), ref.ints(table), ref.ints(free), ref.ints([n_free])
            kv = d_t if in_place else torch.full_like(d_t, -5)
            nf = d_nf if in_place else torch.full_like(d_nf, -5)
            for again in range(1 if in_place else 2):        # out of place the call can be repeated
                pg.tables(d_t, d_n, d_table, d_free, d_nf, q_start.t, kv, slots.t, nf)
            got = (d_table, d_free, nf, q_start.t, kv, slots.t)
            for name, a, b in zip(("table", "free", "n_free", "q_start", "kv_len", "slots"), got, want):
                assert np.array_equal(a.cpu().numpy(), np.asarray(b).reshape(a.shape)), (name, trial, in_place)
        slots.check("slots")
        q_start.check("q_start")
        assert pg.device_status() == 0


def test_tables_flags_bad_lengths_and_stack(fk):
    pg = make(fk, n_pages=8, W=4, B=3)
    i = ref.ints
    table, free = i(np.zeros((3, 4))), i(np.arange(8))
    kv, nf, start, slots = i([0, 0, 0]), i([0]), i([0] * 4), i([0] * 4)
    pg.tables(i([-3, 65, 2]), i([1, 1, 1]), table, free, i([4]), start, kv, slots, nf)
    assert kv.tolist() == [-3, 65, 3] and slots.tolist() == [-1, -1, 2, -1] and pg.device_status() == 0x103
    pg.reset_device_status()
    pg.tables(i([0, 0, 2]), i([1, 1, 1]), table, free, i([99]), start, kv, slots, nf)
    assert pg.device_status() == 0x104 and nf.tolist() == [6]
    pg.reset_device_status()
    free.fill_(1 << 30)
    pg.tables(i([0, 0, 2]), i([1, 0, 1]), table, free, i([4]), start, kv, slots, nf)
    assert slots.tolist() == [-1, 2, -1, -1] and pg.device_status() == 0x101


# ------------------------------------------------------------------------------------------------ store

def _value_classes(rng, n, H):
    x = rng.standard_normal((n, H, 128)) * np.exp(rng.standard_normal((n, H, 1)) * 2.0)
    x[rng.random(x.shape) < 0.05] = 0.0
    return x


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,H,lens,new", [
    (16, 1, [1], [1]),
    (16, 2, [16, 17, 40, 5], [16, 1, 23, 2]),
    (32, 5, [33, 31, 64, 1, 100], [1, 31, 30, 1, 70]),
    (64, 3, [700, 64, 65, 130], [300, 64, 1, 3]),
    (128, 2, [1000, 127, 129], [1000, 5, 2]),
    (16, 2, [300] * 8, [1] * 8),
    (64, 8, [5000, 77], [4000, 77]),        # several tokens a CTA, runs across the tiles
])
def test_store(fk, dtype, page, H, lens, new):
    rng = np.random.default_rng(sum(lens) + page)
    B, W = len(lens), max(ref.pages_of(n, page) for n in lens)
    n_pages = sum(ref.pages_of(n, page) for n in lens) + 2
    table = ref.spread(lens, page, n_pages, W, rng)
    slots = [int(table[b, p // page]) * page + p % page for b in range(B) for p in range(lens[b] - new[b], lens[b])]
    starts = [i for i, s in enumerate(slots) if i == 0 or s != slots[i - 1] + 1 or s % page == 0]
    slots.insert(starts[len(starts) // 2], -1)                           # a token without a slot, not inside a page's run
    n = len(slots)
    pg = make(fk, H=H, page=page, n_pages=n_pages, W=W, B=B, dtype=dtype)
    out = [Guarded((n_pages, H, page, 128), torch.uint8) for _ in range(2)] + [Guarded((n_pages, H), torch.float32) for _ in range(2)]
    before = [ref.random_cache(rng, n_pages, H, page, [a - b for a, b in zip(lens, new)], table) for _ in range(2)]
    wide = torch.zeros((n, H + 1, 128), dtype=dtype, device="cuda")      # token rows of a wider tensor
    xs = []
    for k in range(2):
        x = torch.from_numpy(_value_classes(rng, n, H)).to(dtype)
        xs.append(x.double().numpy())
        out[k].t.copy_(torch.from_numpy(before[k][0]))
        out[2 + k].t.copy_(torch.from_numpy(before[k][1]))
    views = []
    for x in xs:
        w = wide.clone()
        w[:, :H] = torch.from_numpy(x).to(dtype).cuda()
        views.append(w[:, :H])
    codes = [o.t.view(torch.float8_e4m3fn) for o in out[:2]]
    pg.store(views[0], views[1], ref.ints(slots), codes[0], codes[1], out[2].t, out[3].t)
    assert pg.device_status() == 0
    for k in range(2):
        want_c, want_s = ref.store(xs[k], slots, before[k][0], before[k][1], page)
        assert np.array_equal(out[2 + k].t.cpu().numpy().astype(np.float64), want_s)
        wrong = np.argwhere(out[k].t.cpu().numpy() != want_c)
        assert len(wrong) == 0, (len(wrong), wrong[:4], wrong[-4:])
    for o in out:
        o.check("cache")


def test_store_of_values_at_the_edges(fk):
    """Infinities, NaN, zeros, the largest and smallest float32 magnitudes: each head of one page a case of its own."""
    x = np.zeros((3, 8, 128))
    x[:, 0] = np.inf; x[1, 0, 5] = 3.0
    x[:, 1] = np.nan; x[0, 1, 7] = -2.0; x[2, 1, 9] = -np.inf
    x[:, 3] = 3.3e38
    x[:, 4] = 1e-45
    x[:, 5] = 2.0 ** -126 * 448
    x[:, 6, ::2] = 448.0; x[:, 6, 1::2] = -0.4375
    x[:, 7] = np.linspace(-465, 465, 128); x[0, 7, 0] = 449.0
    x32 = torch.from_numpy(x).float()
    pg = make(fk, H=8, page=16, n_pages=2, W=1, B=1, dtype=torch.float32)
    kp, vp, ks, vs = pg.alloc()
    for t in (kp, vp):
        t.view(torch.uint8).fill_(127)
    ks.fill_(float("nan")); vs.fill_(float("nan"))       # a fresh page does not read its old scale
    pg.store(x32.cuda(), x32.cuda(), ref.ints([16, 17, 18]), kp, vp, ks, vs)
    want_c, want_s = ref.store(x32.double().numpy(), [16, 17, 18], np.full((2, 8, 16, 128), 127, np.uint8), np.full((2, 8), np.nan), 16)
    got = kp.view(torch.uint8).cpu().numpy()
    nan = (want_c & 127) == 127
    assert np.array_equal((got & 127) == 127, nan) and np.array_equal(got[~nan], want_c[~nan])
    assert np.array_equal(ks.cpu().numpy().astype(np.float64), want_s, equal_nan=True)
    assert torch.equal(kp.view(torch.uint8), vp.view(torch.uint8))


def test_store_skips_slots_outside_the_pool(fk):
    pg = make(fk, H=1, page=16, n_pages=2, W=2, B=2)
    k = torch.ones(3, 1, 128, dtype=torch.bfloat16, device="cuda")
    kp, vp, ks, vs = pg.alloc()
    for t in (kp, vp):
        t.view(torch.uint8).zero_()
    ks.zero_(); vs.zero_()
    pg.store(k, k, ref.ints([32, 0, 0x7fffffff]), kp, vp, ks, vs)
    assert pg.device_status() == 0x102
    assert kp.float().sum().item() * 2.0 ** -8 == 128 and ks[0, 0].item() == 2.0 ** -8 and ks[1, 0].item() == 0.0


# ------------------------------------------------------------------------------------------------ load

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,H,lens,L", [(16, 1, [1], 1), (32, 3, [0, 100, 33], 101), (64, 2, [640, 1], 64), (128, 4, [129, 500, 128], 700)])
def test_load(fk, dtype, page, H, lens, L):
    rng = np.random.default_rng(sum(lens) + page)
    W = max(1, max(ref.pages_of(n, page) for n in lens))
    n_pages = sum(ref.pages_of(n, page) for n in lens) + 1
    table = ref.spread(lens, page, n_pages, W, rng)
    pg = make(fk, H=H, page=page, n_pages=n_pages, W=W, B=len(lens), dtype=dtype)
    kc, ks = ref.random_cache(rng, n_pages, H, page, lens, table, pow2=False)
    vc, vs = ref.random_cache(rng, n_pages, H, page, lens, table)
    outs = [Guarded((len(lens), H, L, 128), dtype, float("nan")) for _ in range(2)]
    pg.load(ref.ints(lens), ref.ints(table), ref.cuda8(kc), ref.cuda8(vc), ref.cuda32(ks), ref.cuda32(vs), L, outs[0].t, outs[1].t)
    for o, c, s in ((outs[0], kc, ks), (outs[1], vc, vs)):
        want = np.zeros((len(lens), H, L, 128))
        for b, n in enumerate(lens):
            k = min(n, L)
            want[b, :, :k] = ref.rows_of(c, s, table[b], n, page)[:, :k]
        got = o.t.double().cpu().numpy()
        # one rounding of code * scale to the tensor type (float32: the product is rounded once too)
        half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
        assert np.all(np.abs(got - want) <= half * np.abs(want) * (1 + 2.0 ** -20))
        o.check("rows")
    assert pg.device_status() == 0


# ------------------------------------------------------------------------------------------------ attention

def _attn_tol(dtype, want, v_max):
    """Per element.  bf16: the output's rounding, half a step 2^-8 of the value, and 2^-8 of the largest |V| of the head for
    weights held in 8-bit terms (at least two terms: a weight is off by at most 2^-8 of itself, and the weights sum to one).
    float32: 4e-6 of the largest |V|: weights off by 2^-20 of themselves, scores of magnitude below 2^5 off by 2^-24 of
    themselves times the sum's growth, exp2 and the products each a few 2^-24."""
    if dtype == torch.bfloat16:
        return 2.0 ** -8 * np.abs(want) + 2.0 ** -8 * v_max
    return 4e-6 * v_max + 2.0 ** -23 * np.abs(want)


def _attn_case(fk, dtype, page, H, G, lens, new, pad=0, pow2=True, scale=0.0, seed=0, W_extra=0, qmul=1.0):
    rng = np.random.default_rng(sum(lens) + page + G + seed)
    B = len(lens)
    W = max(1, max(ref.pages_of(n, page) for n in lens)) + W_extra
    n_pages = sum(ref.pages_of(n, page) for n in lens) + 2
    table = ref.spread(lens, page, n_pages, W, rng)
    kc, ks = ref.random_cache(rng, n_pages, H, page, lens, table, pow2)
    vc, vs = ref.random_cache(rng, n_pages, H, page, lens, table, pow2)
    n_new = new or [1] * B
    start = np.concatenate([[0], np.cumsum(n_new)])
    n = int(start[-1]) + pad
    q = torch.from_numpy(rng.standard_normal((n, H * G, 128)) * qmul).to(dtype)
    pg = make(fk, H=H, G=G, page=page, n_pages=n_pages, W=W, B=B, dtype=dtype)
    out = Guarded((n, H * G, 128), dtype, 7.0)
    args = (ref.ints(lens), ref.ints(table), ref.cuda8(kc), ref.cuda8(vc), ref.cuda32(ks), ref.cuda32(vs))
    pg.attn(q.cuda(), *args, out.t, q_start=None if new is None else ref.ints(start), scale=scale)
    assert pg.device_status() == 0
    out.check("out")
    want = ref.attn(q.double().numpy(), start, lens, table, kc, ks, vc, vs, page, scale)
    got = out.t.double().cpu().numpy()
    assert np.all(got[int(start[-1]):] == 7.0)                           # padding rows
    for b in range(B):
        V = ref.rows_of(vc, vs, table[b], lens[b], page)
        for h in range(H):
            rows = (slice(start[b], start[b + 1]), slice(h * G, (h + 1) * G))
            w, g = want[rows], got[rows]
            tol = _attn_tol(dtype, w, np.abs(V[h]).max() if lens[b] else 0.0)
            assert np.all(np.abs(g - w) <= tol), (b, h, float((np.abs(g - w) - tol).max()), float(np.abs(g - w).max()))
    return pg, q, args, out, start


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("H,G,lens", [
    (1, 1, [1]), (2, 4, [127, 128, 129, 0, 1]), (3, 7, [300, 17]), (4, 8, [640]), (1, 5, [2500, 3]), (2, 3, [15, 16, 33]),
    (5, 2, [1000, 999]), (1, 6, [257]),
])
def test_decode_attention(fk, dtype, page, H, G, lens):
    _attn_case(fk, dtype, page, H, G, lens, None, pow2=page != 32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,H,G,lens,new,pad", [
    (16, 1, 1, [1], [1], 0),
    (16, 2, 4, [40, 9, 0, 3], [7, 9, 0, 1], 3),          # a sequence without new tokens; padding
    (64, 2, 4, [300, 128, 129], [130, 1, 129], 0),
    (32, 1, 7, [500, 64], [64, 33], 1),
    (128, 1, 8, [200], [200], 0),
    (64, 3, 3, [190, 1], [17, 1], 0),
    (16, 1, 2, [5], [9], 0),                              # more new tokens than cached ones: the first rows see nothing
])
def test_ragged_causal_attention(fk, dtype, page, H, G, lens, new, pad):
    _attn_case(fk, dtype, page, H, G, lens, new, pad)


@pytest.mark.parametrize("page,H,G,lens,new", [
    (64, 1, 4, [5000], [40]),               # few blocks, the cached tokens split
    (16, 2, 4, [3000, 700], [2, 1]),        # at most eight columns a sequence: the narrow form, split
    (128, 8, 8, [900, 260], [100, 250]),
    (32, 1, 1, [2100], [700]),
])
def test_ragged_attention_over_split_caches(fk, page, H, G, lens, new):
    _attn_case(fk, torch.bfloat16, page, H, G, lens, new)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_scale_and_sharp_scores(fk, dtype):
    """A given scale, and queries loud enough for one token to take nearly all the weight."""
    _attn_case(fk, dtype, 16, 2, 4, [300, 70], None, scale=0.3)
    _attn_case(fk, dtype, 64, 1, 4, [1500], None, qmul=8.0)
    _attn_case(fk, dtype, 64, 1, 4, [700], [300], qmul=8.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_of_many_sequences(fk, dtype):
    """More sequences than the decode step's scan has threads, more blocks of new tokens than are shared out evenly, more kv
    heads than warps."""
    rng = np.random.default_rng(8)
    lens = rng.integers(0, 40, 300).tolist()
    _attn_case(fk, dtype, 16, 1, 2, lens, None)
    _attn_case(fk, dtype, 16, 40, 1, [140, 3], None)
    _attn_case(fk, dtype, 16, 20, 2, [140, 3], [130, 2])
    lens = rng.integers(1, 20, 1100).tolist()
    _attn_case(fk, dtype, 16, 1, 1, lens, [min(n, 1 + i % 3) for i, n in enumerate(lens)])      # 8 columns a block
    lens = [n + 2 for n in lens]
    _attn_case(fk, dtype, 16, 1, 4, lens, [3] * len(lens), pad=1)                                # 128 (bf16)


def _cache_from_rows(K, V, page, n_pages, table, lens):
    """Codes and scales of float64 rows [B][H, n, 128], stored as the reference stores them."""
    H = K[0].shape[0]
    kc, vc = [np.full((n_pages, H, page, 128), 127, dtype=np.uint8) for _ in range(2)]
    ks, vs = [np.ones((n_pages, H)) for _ in range(2)]
    for b, n in enumerate(lens):
        slots = [int(table[b, p // page]) * page + p % page for p in range(n)]
        kc, ks = ref.store(K[b].transpose(1, 0, 2), slots, kc, ks, page)
        vc, vs = ref.store(V[b].transpose(1, 0, 2), slots, vc, vs, page)
    return kc, ks, vc, vs


def _attn_on(fk, dtype, page, G, q, start, lens, table, kc, ks, vc, vs, **kw):
    H = kc.shape[1]
    pg = make(fk, H=H, G=G, page=page, n_pages=kc.shape[0], W=table.shape[1], B=len(lens), dtype=dtype)
    out = torch.full((q.shape[0], H * G, 128), 7.0, dtype=dtype, device="cuda")
    pg.attn(q.cuda(), ref.ints(lens), ref.ints(table), ref.cuda8(kc), ref.cuda8(vc), ref.cuda32(ks), ref.cuda32(vs), out,
            q_start=None if start is None else ref.ints(start), **kw)
    return pg, out.double().cpu().numpy()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("new", [None, [150]])
@pytest.mark.parametrize("step", [4.0, 30.0, 200.0, -40.0])
def test_attention_when_scores_climb_along_the_sequence(fk, dtype, new, step):
    """Scores that rise (or fall) by `step` nats per 128 tokens: the running maximum is raised in every tile, from a little
    to far beyond float32's range."""
    rng = np.random.default_rng(int(abs(step)))
    lens, page, G = [900], 32, 4
    table = ref.spread(lens, page, 40, 30, rng)
    K = rng.standard_normal((1, 900, 128)) * 0.1
    K[0, :, 0] = np.repeat(np.arange(900) // 32, 1) * step * math.sqrt(128) / 4.0 / 2.0
    V = rng.standard_normal((1, 900, 128))
    kc, ks, vc, vs = _cache_from_rows([K], [V], page, 40, table, lens)
    n = 1 if new is None else new[0]
    q = torch.from_numpy(rng.standard_normal((n, G, 128)) * 0.1).to(dtype)
    q[:, :, 0] = 2.0
    start = [0, n]
    pg, got = _attn_on(fk, dtype, page, G, q, None if new is None else start, lens, table, kc, ks, vc, vs)
    want = ref.attn(q.double().numpy(), start, lens, table, kc, ks, vc, vs, page)
    assert pg.device_status() == 0
    # scores reach |s| = 27 / 2 * |step| * 2: in float32 each is off by a few 2^-24 of that, and a weight by as much
    s_max = 28 * abs(step)
    tol = _attn_tol(dtype, want, np.abs(ref.rows_of(vc, vs, table[0], 900, page)).max()) * (1 + s_max * 2.0 ** -22 / 4e-6)
    if dtype == torch.bfloat16:
        tol = _attn_tol(dtype, want, np.abs(ref.rows_of(vc, vs, table[0], 900, page)).max()) + s_max * 2.0 ** -22 * 4.5
    assert np.all(np.abs(got - want) <= tol), float((np.abs(got - want) - tol).max())


@pytest.mark.parametrize("new", [None, [3], [70]])
def test_attention_with_nan_in_the_cache_and_the_queries(fk, new):
    """A NaN reaches the rows that see it, and no others: not through a masked key, not through a masked value."""
    rng = np.random.default_rng(5)
    lens, page, G, H = [200], 64, 4, 2
    table = ref.spread(lens, page, 6, 4, rng)
    kc, ks = ref.random_cache(rng, 6, H, page, lens, table)
    vc, vs = ref.random_cache(rng, 6, H, page, lens, table)
    n = 1 if new is None else new[0]
    start = [0, n]
    q = torch.from_numpy(rng.standard_normal((n, H * G, 128))).to(torch.bfloat16)

    def cell(pos):
        return table[0, pos // page], pos % page

    for k_at, v_at in (((150, 199), (140, 199, 170)) if new else ((10,), (60, 199)), ((), (199, 198)), ((199,), ())):
        kc2, vc2 = kc.copy(), vc.copy()
        for pos in k_at:
            p, r = cell(pos)
            kc2[p, 0, r, 3] = 0x7f
        for i, pos in enumerate(v_at):
            p, r = cell(pos)
            vc2[p, 1, r, 10 * i + 1] = 0xff
        pg, got = _attn_on(fk, torch.bfloat16, page, G, q, None if new is None else start, lens, table, kc2, ks, vc2, vs)
        want = ref.attn(q.double().numpy(), start, lens, table, kc2, ks, vc2, vs, page)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        ok = ~np.isnan(want)
        assert np.all(np.abs(got - want)[ok] <= _attn_tol(torch.bfloat16, want, 4.0)[ok])
    q2 = q.clone()
    q2[0, 1, 5] = float("nan")
    q2[n - 1, 6, 9] = float("inf")
    pg, got = _attn_on(fk, torch.bfloat16, page, G, q2, None if new is None else start, lens, table, kc, ks, vc, vs)
    bad = np.zeros(got.shape, dtype=bool)
    bad[0, 1] = True
    bad[n - 1, 6] = True
    assert np.array_equal(np.isnan(got), bad)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_over_pages_of_very_different_scales(fk, dtype):
    """Pages of zeros (the smallest scale), of tiny and of large values side by side."""
    rng = np.random.default_rng(11)
    lens, page, G = [160], 16, 2
    table = ref.spread(lens, page, 12, 10, rng)
    K, V = rng.standard_normal((2, 160, 128)), rng.standard_normal((2, 160, 128))
    V[:, 16:48] = 0.0
    V[:, 64:80] *= 1e-20
    V[0, 80:96] *= 1e3
    K[:, 112:128] = 0.0
    kc, ks, vc, vs = _cache_from_rows([K], [V], page, 12, table, lens)
    for new in (None, [50]):
        n = 1 if new is None else 50
        q = torch.from_numpy(rng.standard_normal((n, 2 * G, 128))).to(dtype)
        pg, got = _attn_on(fk, dtype, page, G, q, None if new is None else [0, n], lens, table, kc, ks, vc, vs)
        want = ref.attn(q.double().numpy(), [0, n], lens, table, kc, ks, vc, vs, page)
        for h in range(2):
            rows = ref.rows_of(vc, vs, table[0], 160, page)[h]
            sl = slice(h * G, (h + 1) * G)
            tol = _attn_tol(dtype, want[:, sl], np.abs(rows).max())
            assert np.all(np.abs(got[:, sl] - want[:, sl]) <= tol)
    V[:] = 0.0                                                       # every value zero: zeros, not NaN
    kc, ks, vc, vs = _cache_from_rows([K], [V], page, 12, table, lens)
    pg, got = _attn_on(fk, dtype, page, G, q, [0, 50], lens, table, kc, ks, vc, vs)
    assert np.all(got == 0.0)


@pytest.mark.parametrize("new", [None, [5], [90]])
def test_attention_skips_pages_outside_the_pool(fk, new):
    rng = np.random.default_rng(3)
    lens, page, G, H = [300], 32, 4, 1
    table = ref.spread(lens, page, 12, 10, rng)
    kc, ks = ref.random_cache(rng, 12, H, page, lens, table)
    vc, vs = ref.random_cache(rng, 12, H, page, lens, table)
    n = 1 if new is None else new[0]
    q = torch.from_numpy(rng.standard_normal((n, G, 128))).to(torch.bfloat16)
    bad = table.copy()
    bad[0, 0], bad[0, 3], bad[0, 5] = 12, -1, 0x7fffffff
    pg, got = _attn_on(fk, torch.bfloat16, page, G, q, None if new is None else [0, n], lens, bad, kc, ks, vc, vs)
    assert pg.device_status() == 0x101
    keep = [p for p in range(300) if p // page not in (0, 3, 5)]
    K = ref.rows_of(kc, ks, table[0], 300, page)[0]
    V = ref.rows_of(vc, vs, table[0], 300, page)[0]
    want = np.zeros_like(got)
    for i in range(n):
        seen = [p for p in keep if p < 300 - n + i + 1]
        for g in range(G):
            s = K[seen] @ q[i, g].double().numpy() / math.sqrt(128)
            w = np.exp(s - s.max())
            want[i, g] = w @ V[seen] / w.sum()
    assert np.all(np.abs(got - want) <= _attn_tol(torch.bfloat16, want, np.abs(V[keep]).max()))
    pg.reset_device_status()
    assert pg.device_status() == 0


def test_lengths_beyond_the_table_are_cut_and_reported(fk):
    rng = np.random.default_rng(4)
    lens, page = [64], 16
    table = ref.spread(lens, page, 6, 4, rng)
    kc, ks = ref.random_cache(rng, 6, 2, page, lens, table)
    vc, vs = ref.random_cache(rng, 6, 2, page, lens, table)
    q = torch.from_numpy(rng.standard_normal((1, 4, 128))).to(torch.bfloat16)
    pg, good = _attn_on(fk, torch.bfloat16, page, 2, q, None, [64], table, kc, ks, vc, vs)
    assert pg.device_status() == 0
    for start in (None, [0, 1]):
        pg, got = _attn_on(fk, torch.bfloat16, page, 2, q, start, [1000], table, kc, ks, vc, vs)
        assert pg.device_status() == 0x103 and np.array_equal(got, good)
        pg, got = _attn_on(fk, torch.bfloat16, page, 2, q, start, [-5], table, kc, ks, vc, vs)
        assert pg.device_status() == 0x103 and np.all(got == 0.0)
    pg, got = _attn_on(fk, torch.bfloat16, page, 2, q, [0, 5], [64], table, kc, ks, vc, vs)
    assert pg.device_status() == 0x105 and np.all(got == 7.0)        # more query rows than there are: none is written
    K, V = pg.load(ref.ints([70]), ref.ints(table), ref.cuda8(kc), ref.cuda8(vc), ref.cuda32(ks), ref.cuda32(vs), 80)
    assert bool((K[:, :, 64:] == 0).all()) and bool((K[0, :, 63] != 0).any())
    bad = table.copy()
    bad[0, 1] = 6
    pg.reset_device_status()
    K, V = pg.load(ref.ints([64]), ref.ints(bad), ref.cuda8(kc), ref.cuda8(vc), ref.cuda32(ks), ref.cuda32(vs), 64)
    assert pg.device_status() == 0x101 and bool((V[:, :, 16:32] == 0).all()) and bool((V[0, :, 40] != 0).any())


def test_cache_offsets_beyond_32_bits(fk):
    """A pool of more than 4 GiB a tensor: pages at its far end are written, read and attended to."""
    H, page, n_pages = 8, 64, 70000
    pg = make(fk, H=H, G=2, page=page, n_pages=n_pages, W=4, B=2)
    kp, vp, ks, vs = pg.alloc()
    rng = np.random.default_rng(9)
    lens = [130, 70]
    table = np.array([[69999, 3, 69990, 0], [65536, 69998, 0, 0]])
    slots = [int(table[b, p // page]) * page + p % page for b in range(2) for p in range(lens[b])]
    k, v = [torch.from_numpy(rng.standard_normal((200, H, 128))).to(torch.bfloat16) for _ in range(2)]
    pg.store(k.cuda(), v.cuda(), ref.ints(slots), kp, vp, ks, vs)
    used = sorted(set(s // page for s in slots))
    at = {p: i for i, p in enumerate(used)}
    small = np.array([[at.get(p, 0) for p in row] for row in table])
    z = np.zeros((len(used), H, page, 128), dtype=np.uint8)
    kc, ksr = ref.store(k.double().numpy(), [at[s // page] * page + s % page for s in slots], z, np.ones((len(used), H)), page)
    vc, vsr = ref.store(v.double().numpy(), [at[s // page] * page + s % page for s in slots], z, np.ones((len(used), H)), page)
    K, V = pg.load(ref.ints(lens), ref.ints(table), kp, vp, ks, vs, 130)
    out = torch.empty((2, H * 2, 128), dtype=torch.bfloat16, device="cuda")
    q = torch.from_numpy(rng.standard_normal((2, H * 2, 128))).to(torch.bfloat16)
    pg.attn(q.cuda(), ref.ints(lens), ref.ints(table), kp, vp, ks, vs, out)
    for b, n in enumerate(lens):
        assert np.array_equal(K[b, :, :n].double().cpu().numpy(), ref.rows_of(kc, ksr, small[b], n, page))   # 4 bits fit bf16
        assert np.array_equal(V[b, :, :n].double().cpu().numpy(), ref.rows_of(vc, vsr, small[b], n, page))
    want = ref.attn(q.double().numpy(), [0, 1, 2], lens, small, kc, ksr, vc, vsr, page)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= _attn_tol(torch.bfloat16, want, 5.0))
    assert pg.device_status() == 0


# ------------------------------------------------------------------------------------------------ calls

def test_strided_queries_streams_workspaces_and_repeats(fk):
    pg, q, args, out, start = _attn_case(fk, torch.bfloat16, 32, 2, 4, [700, 300, 5], None, W_extra=3)
    first = out.t.clone()
    wide = torch.randn(3, 8 + 4, 128, device="cuda").to(torch.bfloat16)
    wide[:, 2:10] = q.cuda()
    again = torch.empty_like(first)
    pg.attn(wide[:, 2:10], *args, again)                             # a slice of a fused projection
    assert torch.equal(first, again)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    on_side = torch.zeros_like(first)
    torch.cuda.synchronize()
    pg.attn(q.cuda(), *args, on_side, stream=side)
    raw = torch.zeros_like(first)
    torch.cuda.synchronize()
    pg.attn(q.cuda(), *args, raw, stream=side.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(first, on_side) and torch.equal(first, raw)
    ws = Guarded((pg.attn_bytes(3, 3),), torch.uint8)
    pg.attn(q.cuda(), *args, again.zero_(), ws=ws.t)
    ws.check("workspace")
    assert torch.equal(first, again)
    # two calls at once, each with a workspace of its own
    outs = [torch.zeros_like(first) for _ in range(8)]
    streams = [torch.cuda.Stream() for _ in range(4)]
    dq = q.cuda()
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        pg.attn(dq, *args, o, stream=streams[i % 4])
    torch.cuda.synchronize()
    assert all(torch.equal(first, o) for o in outs)


def test_refusals(fk):
    pg = make(fk, H=2, G=2, page=16, n_pages=8, W=4, B=2)
    kp, vp, ks, vs = pg.alloc()
    lib, h = fk.load(), pg._h
    i = ref.ints
    kv, table = i([5, 6]), i(np.zeros((2, 4)))
    q = torch.zeros(2, 4, 128, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(2, 2, 128, dtype=torch.bfloat16, device="cuda")
    out, slots, ws = torch.zeros_like(q), i([0, 16]), torch.empty(pg.attn_bytes(2, 2), dtype=torch.uint8, device="cuda")
    before = pg.launch_count()

    def attn(**kw):
        a = dict(q=q.data_ptr(), ld=512, st=None, n=2, b=2, kv=kv.data_ptr(), tb=table.data_ptr(), kp=kp.data_ptr(), vp=vp.data_ptr(),
                 ks=ks.data_ptr(), vs=vs.data_ptr(), scale=0.0, out=out.data_ptr(), ws=ws.data_ptr(), wb=ws.numel())
        a.update(kw)
        return lib.faedkv_pages_attn(h, a["q"], a["ld"], a["st"], a["n"], a["b"], a["kv"], a["tb"], a["kp"], a["vp"], a["ks"], a["vs"],
                                     a["scale"], a["out"], a["ws"], a["wb"], None)

    for kw, code in [(dict(b=3, n=3), -3), (dict(b=0, n=0), -3), (dict(n=1), -3), (dict(n=-1, st=kv.data_ptr()), -3), (dict(ld=511), -3),
                     (dict(ld=516), -5), (dict(q=None), -1), (dict(out=None), -1), (dict(ws=None), -1), (dict(wb=8), -3), (dict(tb=None), -1),
                     (dict(q=q.data_ptr() + 8), -5), (dict(kv=kv.data_ptr() + 2), -5), (dict(scale=-1.0), -1), (dict(scale=math.nan), -1),
                     (dict(scale=math.inf), -1), (dict(n=(1 << 30), st=kv.data_ptr()), -3), (dict(kp=kp.data_ptr() + 4), -5)]:
        assert attn(**kw) == code, kw
    assert b"scale" in lib.faedkv_pages_last_error(h) or lib.faedkv_pages_last_error(h)

    def store(**kw):
        a = dict(k=k.data_ptr(), v=k.data_ptr(), ld=256, s=slots.data_ptr(), n=2)
        a.update(kw)
        return lib.faedkv_pages_store(h, a["k"], a["v"], a["ld"], a["s"], a["n"], kp.data_ptr(), vp.data_ptr(), ks.data_ptr(), vs.data_ptr(), None)

    for kw, code in [(dict(n=-1), -3), (dict(ld=255), -3), (dict(ld=260), -5), (dict(k=None), -1), (dict(s=None), -1), (dict(v=k.data_ptr() + 2), -5)]:
        assert store(**kw) == code, kw
    assert store(n=0) == 0
    t = kv.data_ptr()
    big = i([0] * 4000)
    assert lib.faedkv_pages_tables(h, t, t, 2, table.data_ptr(), big.data_ptr(), t, 3000, big.data_ptr(), t, big.data_ptr(), t, None, None) == -1
    assert lib.faedkv_pages_tables(h, t, t, 5, table.data_ptr(), big.data_ptr(), t, 2, big.data_ptr(), t, big.data_ptr(), t, None, None) == -3
    assert lib.faedkv_pages_tables(h, t, t, 2, table.data_ptr(), big.data_ptr(), t, -2, big.data_ptr(), t, big.data_ptr(), t, None, None) == -3
    assert lib.faedkv_pages_tables(h, None, t, 2, table.data_ptr(), big.data_ptr(), t, 2, big.data_ptr(), t, big.data_ptr(), t, None, None) == -1
    rows = torch.empty(2, 2, 8, 128, dtype=torch.bfloat16, device="cuda")
    r = rows.data_ptr()
    args = (kp.data_ptr(), vp.data_ptr(), ks.data_ptr(), vs.data_ptr())
    assert lib.faedkv_pages_load(h, t, table.data_ptr(), 2, 0, *args, r, r, None) == -3
    assert lib.faedkv_pages_load(h, t, table.data_ptr(), 2, 8, args[0], None, args[2], None, None, None, None) == -1
    assert lib.faedkv_pages_load(h, t, table.data_ptr(), 2, 8, None, None, None, None, None, None, None) == -1
    assert lib.faedkv_pages_load(h, None, table.data_ptr(), 2, 8, *args, r, r, None) == -1
    assert pg.launch_count() == before                               # nothing was launched
    assert lib.faedkv_pages_load(h, t, table.data_ptr(), 2, 8, args[0], None, args[2], None, r, None, None) == 0
    with pytest.raises(ValueError, match="table"):
        pg.attn(q, kv, table[:, :3], kp, vp, ks, vs, out)
    with pytest.raises(ValueError, match="out"):
        pg.attn(q, kv, table, kp, vp, ks, vs, out.float())
    with pytest.raises(ValueError, match="kv_len"):
        pg.attn(q, kv.cpu(), table, kp, vp, ks, vs, out)
    with pytest.raises(ValueError, match="ws"):
        pg.attn(q, kv, table, kp, vp, ks, vs, out, ws=ws[:8])
    with pytest.raises(ValueError, match="same tokens"):
        pg.store(k, k[:1], slots, kp, vp, ks, vs)
    with pytest.raises(fk.FaedkvError) as e:
        pg.attn(torch.zeros(3, 4, 128, dtype=torch.bfloat16, device="cuda"), kv, table, kp, vp, ks, vs,
                torch.zeros(3, 4, 128, dtype=torch.bfloat16, device="cuda"))
    assert e.value.code == -3
    pg.attn(q[:0], kv, table, kp, vp, ks, vs, out[:0], q_start=i([0, 0, 0]))          # no tokens: nothing to do


# ------------------------------------------------------------------------------------------------ a run of them

def _serve(fk, dtype, steps, graph):
    """A small server: three prompts arrive, one joins later, one finishes and its pages are used again; every step is
    tables -> store -> attention.  Returns what the steps gave and the state, and the reference's."""
    H, G, page, W, B, n_pages = 2, 4, 16, 8, 4, 26
    rng = np.random.default_rng(77)
    pg = make(fk, H=H, G=G, page=page, n_pages=n_pages, W=W, B=B, dtype=dtype)
    kp, vp, ks, vs = pg.alloc()
    for t in (kp, vp):
        t.view(torch.uint8).fill_(127)
    ks.fill_(1.0); vs.fill_(1.0)
    kc, vc = [np.full((n_pages, H, page, 128), 127, dtype=np.uint8) for _ in range(2)]
    ksr, vsr = np.ones((n_pages, H)), np.ones((n_pages, H))
    t_len, table = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.full((B, W), -1, dtype=torch.int32, device="cuda")
    free, n_free = ref.ints(np.arange(n_pages)), ref.ints([n_pages])
    state = ([0] * B, [[-1] * W for _ in range(B)], list(range(n_pages)), n_pages)
    plan = [[37, 20, 1, 0], [1, 1, 1, 0], [1, 1, 1, 55], [1, -1, 1, 1], [1, 33, 1, 1]] + [[1, 1, 1, 1]] * steps
    most = 64
    # buffers of the largest step: what a captured step works on
    n_new, q_start, slots = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B + 1, dtype=torch.int32, device="cuda"), None
    got, want = [], []
    dec = {"k": torch.zeros((B, H, 128), dtype=dtype, device="cuda"), "v": torch.zeros((B, H, 128), dtype=dtype, device="cuda"),
           "q": torch.zeros((B, H * G, 128), dtype=dtype, device="cuda"), "out": torch.zeros((B, H * G, 128), dtype=dtype, device="cuda"),
           "slots": torch.zeros(B, dtype=torch.int32, device="cuda")}
    captured = None

    def decode_step():
        pg.tables(t_len, n_new, table, free, n_free, q_start, t_len, dec["slots"], n_free)
        pg.store(dec["k"], dec["v"], dec["slots"], kp, vp, ks, vs)
        pg.attn(dec["q"], t_len, table, kp, vp, ks, vs, dec["out"])

    for step, new in enumerate(plan):
        n = sum(max(x, 0) for x in new)
        pad = 0 if step >= 5 else 2
        k, v = [torch.from_numpy(rng.standard_normal((n + pad, H, 128)) * np.exp(rng.standard_normal((n + pad, 1, 1)))).to(dtype) for _ in range(2)]
        q = torch.from_numpy(rng.standard_normal((n + pad, H * G, 128))).to(dtype)
        n_new.copy_(ref.ints(new))
        if step < 5:
            slots = torch.zeros(n + pad, dtype=torch.int32, device="cuda")
            out = torch.full_like(q.cuda(), 7.0)
            pg.tables(t_len, n_new, table, free, n_free, q_start, t_len, slots, n_free)
            pg.store(k.cuda(), v.cuda(), slots, kp, vp, ks, vs)
            pg.attn(q.cuda(), t_len, table, kp, vp, ks, vs, out, q_start=q_start)
        else:
            dec["k"].copy_(k); dec["v"].copy_(v); dec["q"].copy_(q)
            if not graph:
                decode_step()
            elif captured is None:
                torch.cuda.synchronize()
                captured = torch.cuda.CUDAGraph()
                with torch.cuda.graph(captured):
                    decode_step()
                captured.replay()
            else:
                captured.replay()
            out = dec["out"]
        torch.cuda.synchronize()
        got.append(out.clone())
        tb, fr, nf, st, kv, sl = ref.tables(state[0], new, state[1], state[2], state[3], n + pad, page)
        kc, ksr = ref.store(k.double().numpy(), sl, kc, ksr, page)
        vc, vsr = ref.store(v.double().numpy(), sl, vc, vsr, page)
        want.append((ref.attn(q.double().numpy(), st, kv, tb, kc, ksr, vc, vsr, page), st, new))
        state = (kv, tb, fr, nf)
    return pg, got, want, state, (t_len, table, n_free), (kp, vp, ks, vs), (kc, ksr, vc, vsr)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_served_run_against_the_reference(fk, dtype):
    pg, got, want, state, dev, cache, refs = _serve(fk, dtype, 20, graph=False)
    kv, tb, fr, nf = state
    assert dev[0].tolist() == kv and dev[2].tolist() == [nf]
    for b in range(4):
        n = ref.pages_of(kv[b], 16)
        assert dev[1][b, :n].tolist() == tb[b][:n]
    assert np.array_equal(cache[0].view(torch.uint8).cpu().numpy(), refs[0]) and np.array_equal(cache[1].view(torch.uint8).cpu().numpy(), refs[2])
    for g, (w, st, new) in zip(got, want):
        g = g.double().cpu().numpy()
        for b in range(4):
            rows = slice(st[b], st[b + 1])
            # |V| up to 4.5 standard deviations times e^{4.5}: the largest stored magnitude bounds it
            assert np.all(np.abs(g[rows] - w[rows]) <= _attn_tol(dtype, w[rows], np.abs(ref.VALUES[refs[2][refs[2] != 127]]).max() * refs[3].max()))
    assert pg.device_status() == 0


def test_a_captured_step_equals_the_eager_one(fk):
    eager = _serve(fk, torch.bfloat16, 20, graph=False)
    graph = _serve(fk, torch.bfloat16, 20, graph=True)
    for a, b in zip(eager[1], graph[1]):
        assert torch.equal(a, b)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(eager[5], graph[5]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_cached_tokens_go_on_to_the_frequency_domain(fk, oracle, dtype):
    """Rows out of the pages feed the prefill transform; with every bin kept, reconstruction gives them back."""
    H, page, T = 2, 32, 256
    pg = make(fk, H=H, G=2, page=page, n_pages=9, W=8, B=1, dtype=dtype)
    rng = np.random.default_rng(2)
    k, v = [torch.from_numpy(rng.standard_normal((T, H, 128))).to(dtype).cuda() for _ in range(2)]
    table = ref.spread([T], page, 9, 8, rng)
    slots = [int(table[0, p // page]) * page + p % page for p in range(T)]
    cache = pg.alloc()
    pg.store(k, v, ref.ints(slots), *cache)
    K, V = pg.load(ref.ints([T]), ref.ints(table), *cache, T)
    # one rounding to e4m3: half a step, 2^-4 of a value above the subnormal range
    diff = (K[0].transpose(0, 1).double() - k.double()).abs()
    assert bool((diff <= k.double().abs() * 2.0 ** -4 + 2.0 ** -10 * cache[2].max().item()).all())
    ctx = fk.Context(n_layers=1, n_kv_heads=H, n_q_heads=2 * H, n_dft=T, max_batch=1, kv_dtype=pg.kv_dtype)
    ctx.plan(0, np.ones(T // 2 + 1, dtype=np.uint8))
    cK, cV = ctx.alloc_coef(0, 1), ctx.alloc_coef(0, 1)
    t_len = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx.compress_prefill(0, K, V, cK, cV, t_len)
    Ko, Vo = torch.empty_like(K), torch.empty_like(V)
    ctx.reconstruct(0, cK, cV, t_len, T, Ko, Vo)
    from helpers import REL_L2_BF16, REL_L2_F32, rel_l2, to_np64
    tol = REL_L2_F32 if dtype == torch.float32 else REL_L2_BF16
    assert rel_l2(to_np64(Ko), to_np64(K)) <= tol and rel_l2(to_np64(Vo), to_np64(V)) <= tol
    # attention over the pages and over the reconstruction of the rows are the same attention
    q = torch.from_numpy(rng.standard_normal((1, 2 * H, 128))).to(dtype).cuda()
    a, b = torch.empty_like(q), torch.empty_like(q)
    pg.attn(q, ref.ints([T]), ref.ints(table), *cache, a)
    ctx.decode_attn(0, q, cK, cV, t_len, b)
    torch.cuda.synchronize()
    bound = 2e-2 if dtype == torch.bfloat16 else 1e-3
    assert float((a.double() - b.double()).abs().max()) <= bound
    ctx.close()
