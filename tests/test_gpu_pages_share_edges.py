"""Shared pages and differential attention at the edges of what their calls accept: starts that are any int32, steps without
forks, every wrong table entry."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import pages_ref as ref
import test_gpu_pages_share as share_tests
from helpers import Guarded
from test_gpu_pages_diff import case as diff_case, expect
from test_gpu_pages_shared import case as shared_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fk():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2507_20030_b200 import binding, build
    build.build()
    binding.load()
    return binding


BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
MOST, LEAST = 2 ** 31 - 1, -2 ** 31


@BOTH
@pytest.mark.parametrize("G", [2, 5, 8])
@pytest.mark.parametrize("starts", [
    [0, 4, MOST, 5, 8],                                     # the search for a block passes the largest int32
    [0, 4, MOST, MOST, MOST],
    [0, 4, LEAST, LEAST, LEAST],
    [LEAST, 0, 4, MOST, MOST],
    [MOST, LEAST, MOST, 0, 4],
])
def test_groups_beside_starts_that_are_no_rows(fk, dtype, G, starts):
    """Whatever stands beside them: rows of no group, and of one whose bounds are not rows, are attended alone."""
    g = [(64, [70, 80, 64, 90]), (128, [130, 140, 150, 129])]
    shared_case(fk, dtype, 16, 2, G, g, starts=starts, shared=[64, 64, 64, 64], status=0x105)


@pytest.mark.parametrize("B", [4, 4096, 4097, 5000])
def test_a_step_without_forks(fk, B):
    """On either side of the batch from which forks are planned ahead of the copies: the height goes through, nothing else changes."""
    pg = fk.Pages(n_kv_heads=1, n_q_heads=1, page_size=16, n_pages=40, max_pages=3, max_batch=B)
    cache = pg.alloc()
    none, free = torch.empty(0, dtype=torch.int32, device="cuda"), ref.ints(np.arange(40)[::-1].copy())
    kv, table = ref.ints(np.arange(B) % 48), ref.ints(np.arange(3 * B).reshape(B, 3) % 40)
    kv0, table0 = kv.clone(), table.clone()
    nf, out = ref.ints([17]), ref.ints([-1])
    pg.fork(none, none, kv, table, free, nf, out, *cache)
    pg.fork(none, none, kv, table, free, nf, nf, *cache, length=none)
    assert out.tolist() == [17] and nf.tolist() == [17] and pg.device_status() == 0
    assert torch.equal(kv, kv0) and torch.equal(table, table0)


@pytest.mark.parametrize("W,B", [(3, 2), (300, 40), (3, 600), (9000, 9)])        # the runs' registers, one and more of a warp; read again
@pytest.mark.parametrize("bad", [-1, -2, -3, LEAST, MOST, 50])
def test_release_flags_every_entry_that_is_no_page(fk, W, B, bad):
    pg = fk.Pages(n_kv_heads=1, n_q_heads=1, page_size=16, n_pages=50, max_pages=W, max_batch=B)
    for row in (0, B - 1):
        for n_new, want in ((-1, [7, 3, 6]), (1, [7])):
            table = np.full((B, W), bad)
            table[row, :3] = [3, bad, 6]                       # the other rows are empty
            kv, nn = np.zeros(B, dtype=np.int64), np.zeros(B, dtype=np.int64)
            kv[row], nn[row] = 40, n_new
            free, nf, out = ref.ints([7] + [-9] * 49), ref.ints([1]), ref.ints(np.zeros(B))
            pg.release(ref.ints(kv), ref.ints(nn), ref.ints(table), free, nf, out, nf)
            assert free.tolist()[:nf.item()] == want and set(free.tolist()[nf.item():]) == {-9}
            assert out[row].item() == (0 if n_new < 0 else 40) and pg.device_status() == 0x101
            pg.reset_device_status()


def diff_call(fk, dtype, page, H, G, lens, new, edit, gain, eps, width=1, scale=None, seed=0):
    """attn_diff over a random cache that edit(rng, table, kc, ks, vc, vs) has changed, against 64 bits row by row."""
    rng = np.random.default_rng(sum(lens) + page + H + 7 * G + seed)
    B, counts = len(lens), new or [1] * len(lens)
    W = max(ref.pages_of(n, page) for n in lens) + width
    n_pages = sum(ref.pages_of(n, page) for n in lens) + 2
    table = ref.spread(lens, page, n_pages, W, rng)
    (kc, ks), (vc, vs) = [ref.random_cache(rng, n_pages, H, page, lens, table) for _ in range(2)]
    edit(rng, table, kc, ks, vc, vs)
    pg = fk.Pages(n_kv_heads=H, n_q_heads=H * G, page_size=page, n_pages=n_pages, max_pages=W, max_batch=B,
                  kv_dtype=fk.BF16 if dtype == torch.bfloat16 else fk.F32)
    q = torch.from_numpy(rng.standard_normal((sum(counts), H * G, 128))).to(dtype).cuda()
    lam = torch.from_numpy(rng.uniform(0.2, 0.8, H * G)).float().cuda()
    gain = torch.from_numpy(rng.uniform(0.5, 1.5, 128)).float().cuda() if gain else None
    out = torch.full_like(q, 7.0)
    start = np.concatenate([[0], np.cumsum(counts)])
    pg.attn_diff(q, ref.ints(lens), ref.ints(table), ref.cuda8(kc), ref.cuda8(vc), ref.cuda32(ks), ref.cuda32(vs), lam, out,
                 q_start=None if new is None else ref.ints(start), gain=gain, eps=eps)
    kind = "f32" if dtype == torch.float32 else "wide" if new is not None else "bf16"
    for b in range(B):
        K, V = [torch.from_numpy(ref.rows_of(c, s, table[b], lens[b], page)).cuda() for c, s in ((kc, ks), (vc, vs))]
        rows = slice(start[b], start[b + 1])
        seen = lens[b] - counts[b] + 1 + torch.arange(counts[b], device="cuda")
        for h in range(H):
            hs = slice(h * G, (h + 1) * G)
            expect(out[rows, hs], kind, q[rows, hs], K[h], V[h], seen, 0.125, lam[hs], gain, eps, (b, h))
    assert pg.device_status() == 0


@BOTH
@pytest.mark.parametrize("exponent", [-100, -75, -50, 0, 50, 70, 100])
@pytest.mark.parametrize("eps", [0.0, 1e-5])
def test_the_norm_of_heads_whose_squares_are_beyond_float32(fk, dtype, exponent, eps):
    """Values of 2^exponent: their squares are no float32, the head over its root mean square is of order one (or, where eps is more, a float32 still)."""
    def edit(rng, table, kc, ks, vc, vs):
        vs *= 2.0 ** exponent
    diff_call(fk, dtype, 16, 2, 2, [300, 17, 129], None, edit, True, eps)                      # decode
    diff_call(fk, dtype, 16, 1, 2, [40, 9], [7, 9], edit, True, eps)                           # new tokens, eight columns
    if dtype == torch.bfloat16:
        diff_call(fk, dtype, 64, 2, 2, [700, 300], [100, 20], edit, True, eps, width=60000)    # columns as rows, two row tiles and one
        diff_call(fk, dtype, 64, 1, 4, [5000], [10], edit, True, eps, width=20000)             # split, one row tile


def test_workspace_of_a_long_differential_prompt(fk):
    """The form with rows keeps no maps: its workspace does not grow with the tokens, and no byte behind it is touched."""
    pg = fk.Pages(n_kv_heads=8, n_q_heads=32, page_size=64, n_pages=4096, max_pages=2048, max_batch=4)
    parts = 148 * 2 * 256 * 130 * 4                            # two partial results of 256 columns a CTA
    assert all(0 < pg.attn_diff_bytes(b, n) <= parts + (1 << 20) for b in (1, 4) for n in (100, 1000, 32768, 131072))
    for b, n in ((4, 4), (4, 2), (1, 1)):                      # eight columns at a time: a float32 row for each token, head and map
        assert pg.attn_diff_bytes(b, n) >= n * 32 * 2 * 128 * 4


@pytest.mark.parametrize("dtype,lens,new,width", [
    (torch.bfloat16, [700, 300], [100, 20], 60000), (torch.bfloat16, [9, 30], [7, 9], 1), (torch.bfloat16, [1200] * 30, [40] * 30, 60000),
    (torch.float32, [700, 300], [100, 20], 1), (torch.bfloat16, [700, 300], None, 1),
])
def test_differential_calls_stay_within_their_workspace(fk, dtype, lens, new, width):
    pg, args, kw, out = diff_case(fk, dtype, 16, 1, 2, lens, new, width=width)
    ws = Guarded((pg.attn_diff_bytes(len(lens), out.shape[0]),), torch.uint8, 255)
    want = out.clone()
    out.fill_(7.0)
    pg.attn_diff(*args, **kw, ws=ws.t)
    ws.check("the workspace")
    assert torch.equal(out, want) and pg.device_status() == 0


@pytest.fixture()
def partition(fk):
    """Handles as on a part of a GPU that has no room for clusters of sixteen CTAs."""
    def pages(**kw):
        pg = fk.Pages(**kw)
        pg.test_cluster(8)
        return pg
    return SimpleNamespace(Pages=pages, BF16=fk.BF16, F32=fk.F32)


@pytest.mark.parametrize("page,W,B,n_pages", [(16, 30, 7, 200), (64, 9, 300, 1500), (64, 2, 256, 700), (64, 2, 257, 700), (16, 257, 200, 20000), (16, 2, 20000, 30000),
                                              (16, 6000, 40, 9000), (16, 9, 30, 65537)])
def test_release_by_clusters_of_eight(partition, page, W, B, n_pages):
    share_tests.test_release(partition, page, W, B, n_pages)


@pytest.mark.parametrize("H,page,W,B,n_pages", [(1, 16, 9, 6, 100), (1, 16, 50, 1500, 66000)])
def test_compact_by_clusters_of_eight(partition, H, page, W, B, n_pages):
    share_tests.test_compact(partition, H, page, W, B, n_pages)


def test_what_room_a_gpu_has_is_asked_for_under_capture_too(fk):
    pg = share_tests.make(fk, n_pages=70000, W=9, B=3)                 # the first call of the handle is a captured one
    cache = pg.alloc()
    t, n_new, table = ref.ints([20, 40, 3]), ref.ints([1, -1, 0]), ref.ints(np.arange(27).reshape(3, 9) + 60000)
    free, nf, new_id = ref.ints(np.zeros(70000)), ref.ints([5]), ref.ints(np.zeros(70000))
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (pg._bytes("faedkv_pages_release_bytes"), pg._bytes("faedkv_pages_compact_bytes"))]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pg.release(t, n_new, table, free, nf, t, nf, ws=ws[0])
        pg.compact(t, table, table, free, nf, new_id, *cache, ws=ws[1])
    assert nf.tolist() == [5]
    graph.replay()
    assert nf.tolist() == [70000 - 3] and t.tolist() == [20, 0, 3] and table[0, :2].tolist() == [0, 1] and table[2, 0].item() == 2
    for bad in (-1, 1, 7, 9, 16):
        with pytest.raises(fk.FaedkvError):
            pg.test_cluster(bad)
