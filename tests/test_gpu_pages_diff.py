"""Differential attention over the paged 8-bit cache on the GPU against its formula in 64 bits."""
import math

import numpy as np
import pytest
import torch

import pages_ref as ref
import pages_share_ref as share
from attn_bounds import attention, close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fk():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2507_20030_b200 import binding, build
    build.build()
    binding.load()
    return binding


def expect(got, kind, q, K, V, seen, scale, lam, gain, eps, what):
    """got, q [m, G, 128] of one kv head.  The difference of the maps adds their errors, and rounds three times in float32; the
    norm moves by no more than the root mean square of what its argument moves by."""
    for g in range(q.shape[1]):
        maps = [attention(kind, q[:, g, part], K[:, part], V, seen, scale) for part in (slice(0, 64), slice(64, 128))]
        (a1, e1), (a2, e2) = maps
        lm = float(lam[g])
        o, e = a1 - lm * a2, e1 + abs(lm) * e2 + 3 * 2.0 ** -24 * (a1.abs() + abs(lm) * a2.abs())
        if gain is not None:
            r = ((o * o).mean(dim=1, keepdim=True) + eps).sqrt()
            er = (torch.as_tensor(e).expand_as(o) ** 2).mean(dim=1, keepdim=True).sqrt() + 2.0 ** -21 * r
            least = torch.where(r > 0, r - er, torch.ones_like(r))
            assert bool((least > 0).all()), "the case leaves nothing to normalise"
            r = torch.where(r > 0, r, torch.ones_like(r))
            w = gain.double()
            o, e = o / r * w, w.abs() * (e / least + o.abs() * er / (r * least)) + 2.0 ** -21 * (o / r * w).abs()
        close(got[:, g], o, e, what)


def case(fk, dtype, page, H, G, lens, new=None, pad=0, gain=True, eps=1e-5, scale=None, lam=None, qmul=1.0, pow2=True, strided=False, seed=0, width=1):
    rng = np.random.default_rng(sum(lens) + page + H * 31 + G + seed)
    B = len(lens)
    W = max(1, max(ref.pages_of(n, page) for n in lens)) + width
    n_pages = sum(ref.pages_of(n, page) for n in lens) + 2
    table = ref.spread(lens, page, n_pages, W, rng)
    (kc, ks), (vc, vs) = [ref.random_cache(rng, n_pages, H, page, lens, table, pow2) for _ in range(2)]
    pg = fk.Pages(n_kv_heads=H, n_q_heads=H * G, page_size=page, n_pages=n_pages, max_pages=W, max_batch=B,
                  kv_dtype=fk.BF16 if dtype == torch.bfloat16 else fk.F32)
    counts = new or [1] * B
    n = sum(counts) + pad
    wide = torch.from_numpy(rng.standard_normal((n, 3 * H * G, 128)) * qmul).to(dtype).cuda()
    q = wide[:, H * G:2 * H * G] if strided else wide[:, :H * G].contiguous()
    lam = torch.as_tensor(rng.uniform(0.2, 0.8, H * G) if lam is None else lam, dtype=torch.float32).cuda()
    gain = torch.from_numpy(rng.uniform(0.5, 1.5, 128)).float().cuda() if gain else None
    out = torch.full((n, H * G, 128), 7.0, dtype=dtype, device="cuda")
    start = np.concatenate([[0], np.cumsum(counts)])
    args = (q, ref.ints(lens), ref.ints(table), ref.cuda8(kc), ref.cuda8(vc), ref.cuda32(ks), ref.cuda32(vs), lam, out)
    kw = dict(q_start=None if new is None else ref.ints(start), gain=gain, eps=eps, scale=scale or 0.0)
    pg.attn_diff(*args, **kw)
    kind = "f32" if dtype == torch.float32 else "wide" if new is not None and n * 2 * G > 8 * B else "bf16"    # (the wider of the two forms' bounds)
    for b in range(B):
        K, V = [torch.from_numpy(ref.rows_of(c, s, table[b], lens[b], page)).cuda() for c, s in ((kc, ks), (vc, vs))]
        m = counts[b]
        seen = lens[b] - m + 1 + torch.arange(m, device="cuda")
        for h in range(H):
            hs = slice(h * G, (h + 1) * G)
            expect(out[start[b]:start[b + 1], hs], kind, q[start[b]:start[b + 1], hs], K[h], V[h], seen, scale or 0.125, lam[hs], gain, eps,
                   (b, h))
    assert bool((out[start[-1]:] == 7.0).all()), "rows of no sequence are left as they were"
    assert pg.device_status() == 0
    return pg, args, kw, out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,H,G,lens", [
    (16, 1, 1, [1]), (32, 2, 4, [127, 128, 129, 0, 1]), (64, 3, 3, [300, 17]), (128, 4, 4, [640]), (16, 1, 2, [2500, 3]),
    (64, 5, 2, [1000, 999]), (32, 8, 1, [257, 40, 33, 1]),
])
@pytest.mark.parametrize("gain", [True, False])
def test_decode(fk, dtype, page, H, G, lens, gain):
    case(fk, dtype, page, H, G, lens, gain=gain, pow2=page != 32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,H,G,lens,new,pad", [
    (16, 1, 1, [1], [1], 0),
    (16, 2, 4, [40, 9, 0, 3], [7, 9, 0, 1], 3),          # a sequence without new tokens; padding
    (64, 2, 2, [300, 128, 129], [130, 1, 129], 0),
    (32, 1, 3, [500, 64], [64, 33], 1),
    (128, 1, 4, [200], [200], 0),
    (16, 1, 2, [5], [9], 0),                              # more new tokens than cached ones: the first rows see nothing
    (64, 1, 4, [3000, 2], [2, 1], 0),
])
def test_new_tokens(fk, dtype, page, H, G, lens, new, pad):
    case(fk, dtype, page, H, G, lens, new, pad)
    case(fk, dtype, page, H, G, lens, new, pad, gain=False, strided=True)
    for gain in (True, False) if dtype == torch.bfloat16 else ():            # wide tables: the form with query columns as rows, where there are many
        case(fk, dtype, page, H, G, lens, new, pad, gain=gain, strided=gain, width=60000)


@pytest.mark.parametrize("page,H,G,lens,new", [
    (64, 1, 4, [5000], [40]),               # few blocks, the cached tokens split over CTAs: two row tiles
    (16, 2, 2, [3000, 700], [20, 3]),       # one row tile, split
    (128, 3, 4, [1900, 260], [100, 250]),
    (32, 1, 1, [2100], [700]),
    (64, 8, 1, [129, 4000], [129, 33]),
])
def test_new_tokens_over_split_caches(fk, page, H, G, lens, new):
    case(fk, torch.bfloat16, page, H, G, lens, new, width=20000)
    case(fk, torch.bfloat16, page, H, G, lens, new, gain=False, width=20000, qmul=4.0)


@pytest.mark.parametrize("page,H,G,lens,new", [
    (64, 2, 4, [30000, 30000], [40, 40]),    # a block of 64 columns behind one of 256, on one CTA
    (16, 2, 4, [4000, 2600, 5000], [36, 70, 33]),
    (32, 1, 2, [9000], [130]),
])
@pytest.mark.parametrize("gain", [True, False])
def test_blocks_of_one_row_tile_behind_blocks_of_two(fk, page, H, G, lens, new, gain):
    """A CTA goes from a block with two row tiles on to one with a single one, whose values have more room: again and again, the same bits."""
    pg, args, kw, out = case(fk, torch.bfloat16, page, H, G, lens, new, 2, gain=gain, width=60000)
    first = out.clone()
    for _ in range(10):
        out.fill_(7.0)
        pg.attn_diff(*args, **kw)
        assert torch.equal(out, first)


def test_more_blocks_than_are_shared_out(fk):
    rng = np.random.default_rng(2)
    lens = rng.integers(1, 20, 1100).tolist()
    for dtype in (torch.bfloat16, torch.float32):
        case(fk, dtype, 16, 1, 1, lens)
        case(fk, dtype, 16, 1, 2, lens, [min(n, 1 + i % 3) for i, n in enumerate(lens)], 2)
    case(fk, torch.bfloat16, 16, 1, 1, [n + 9 for n in lens], [10] * 1100, width=3000)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_scale_lambda_and_eps(fk, dtype):
    case(fk, dtype, 16, 2, 2, [300, 70], scale=0.3)
    case(fk, dtype, 16, 2, 2, [300, 70], lam=[0.0, 1.0, -0.5, 3.0])
    case(fk, dtype, 64, 1, 4, [1500], qmul=8.0)
    case(fk, dtype, 64, 1, 2, [700], [300], qmul=6.0, strided=True)
    case(fk, dtype, 64, 1, 2, [700], [300], qmul=6.0, width=9000)
    case(fk, dtype, 16, 1, 2, [0, 33], eps=0.0)                            # a row of zeros stays one
    case(fk, dtype, 16, 1, 2, [33, 3], eps=10.0)


def test_nothing_of_one_map_without_its_weight(fk):
    """lam = 0 is softmax attention over the first half: equal to attn() of queries whose second half is zero, at the same scale."""
    pg, args, kw, out = case(fk, torch.bfloat16, 16, 2, 4, [300, 70, 1], lam=[0.0] * 8, gain=False)
    q = args[0].clone()
    q[..., 64:] = 0
    plain = torch.empty_like(out)
    pg.attn(q, *args[1:7], plain, scale=0.125)
    # the same columns at the same places but for others beside them: the running reference may differ, and with it a rounding
    assert float((plain.double() - out.double()).abs().max()) <= 2.0 ** -6 * float(plain.double().abs().max())


@pytest.mark.parametrize("which", [0, 1])
def test_nan_reaches_the_rows_that_see_it(fk, which):
    """A NaN value reaches its channel of the rows that see it; a NaN key all channels of them, whichever half it stands in."""
    rng = np.random.default_rng(5)
    page, n, H, G, m = 16, 40, 1, 2, 9
    table = ref.spread([n], page, 4, 3, rng)
    (kc, ks), (vc, vs) = [ref.random_cache(rng, 4, H, page, [n], table) for _ in range(2)]
    at = n - 4                                                 # seen by the last four tokens
    (kc, vc)[which][table[0, at // page], 0, at % page, 70] = 127
    for new, width in ((None, 3), ([m], 3), ([m], 200000)):
        table = np.concatenate([table[:, :3], np.full((1, width - 3), 0x7fffffff)], axis=1)
        pg = fk.Pages(n_kv_heads=H, n_q_heads=G, page_size=page, n_pages=4, max_pages=width, max_batch=1)
        rows = m if new else 1
        q = torch.from_numpy(rng.standard_normal((rows, G, 128))).bfloat16().cuda()
        out = torch.full((rows, G, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        pg.attn_diff(q, ref.ints([n]), ref.ints(table), ref.cuda8(kc), ref.cuda8(vc), ref.cuda32(ks), ref.cuda32(vs),
                     torch.full((G,), 0.5, device="cuda"), out, q_start=ref.ints([0, m]) if new else None)
        nan = torch.isnan(out)
        want = torch.zeros_like(nan)
        sees = slice(rows - 4, rows) if new else slice(0, 1)
        if which:
            want[sees, :, 70] = True
        else:
            want[sees] = True
        assert torch.equal(nan, want)


def test_captured_and_on_another_stream(fk):
    pg, args, kw, out = case(fk, torch.bfloat16, 64, 2, 2, [700, 130, 1])
    want = out.clone()
    side = torch.cuda.Stream()
    ws = torch.empty(pg.attn_diff_bytes(3, 3), dtype=torch.uint8, device="cuda")
    q0 = args[0].clone()
    args[0].zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        args[0].copy_(q0)
        pg.attn_diff(*args, **kw)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pg.attn_diff(*args, **kw, ws=ws)
    for _ in range(3):
        out.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_refusals(fk):
    pg, args, kw, out = case(fk, torch.bfloat16, 16, 2, 2, [33, 5])
    lib, z, n0 = fk.load(), None, pg.launch_count()
    p = [x.data_ptr() for x in args]
    ws = torch.empty(pg.attn_diff_bytes(2, 2), dtype=torch.uint8, device="cuda")
    good = [pg._h, p[0], 512, z, 2, 2, p[1], p[2], p[3], p[4], p[5], p[6], 0.0, p[7], z, 0.0, p[8], ws.data_ptr(), ws.numel(), z]
    for k in (1, 6, 7, 8, 9, 10, 11, 13, 16, 17):
        assert lib.faedkv_pages_attn_diff(*good[:k], z, *good[k + 1:]) == -1, k
        assert lib.faedkv_pages_attn_diff(*good[:k], good[k] + 2, *good[k + 1:]) == -5, k
    for k, bad, code in [(2, 511, -3), (2, 515, -5), (4, 3, -3), (4, -1, -3), (5, 3, -3), (5, 0, -3), (12, -1.0, -1), (12, math.inf, -1), (12, math.nan, -1),
                         (14, p[7] + 4, -5), (15, -1.0, -1), (15, math.nan, -1), (18, ws.numel() - 1, -3)]:
        assert lib.faedkv_pages_attn_diff(*good[:k], bad, *good[k + 1:]) == code, (k, bad)
    five = fk.Pages(n_kv_heads=2, n_q_heads=10, page_size=16, n_pages=4, max_pages=4, max_batch=2)
    assert lib.faedkv_pages_attn_diff(five._h, *good[1:]) == -4 and lib.faedkv_pages_attn_diff_bytes(five._h, 2, 2) == 0
    assert pg.launch_count() == n0 and five.launch_count() == 0
    q, kv, table, kp, vp, ks, vs, lam, _ = args
    for name, bad in (("lam", lam.double()), ("lam", lam[:3]), ("gain", torch.ones(64, device="cuda")), ("out", out[:1]), ("q", q.float())):
        a = dict(zip(("q", "kv_len", "table", "k_pages", "v_pages", "k_scale", "v_scale", "lam", "out"), args))
        with pytest.raises(ValueError, match=name):
            pg.attn_diff(**{**a, name: bad})
    assert pg.launch_count() == n0


def test_against_the_plain_restatement(fk):
    """The same formula in numpy loops, one small case."""
    pg, args, kw, out = case(fk, torch.float32, 16, 2, 2, [20, 3], [4, 1])
    q, kv, table, kp, vp, ks, vs, lam, _ = args
    codes = [x.view(torch.uint8).cpu().numpy() for x in (kp, vp)]
    want, _ = share.attn_diff(q.double().cpu().numpy(), kw["q_start"].tolist(), kv.tolist(), table.tolist(), codes[0], ks.double().cpu().numpy(),
                              codes[1], vs.double().cpu().numpy(), 16, lam.tolist(), kw["gain"].double().cpu().numpy(), 1e-5)
    assert np.abs(out.double().cpu().numpy() - want).max() <= 2.0 ** -15 * np.abs(want).max()
