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
