"""Shared pages on the GPU against the plain reference: fork, release, compact, and the life of requests that share pages."""
import numpy as np
import pytest
import torch

import pages_ref as ref
import pages_share_ref as share
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


def _pool(rng, n_pages, H, page):
    """Any bytes and any scales: a page is moved as it is."""
    codes = [rng.integers(0, 256, (n_pages, H, page, 128), dtype=np.uint8) for _ in range(2)]
    scales = [rng.random((n_pages, H)).astype(np.float32) for _ in range(2)]
    return codes, scales


class Cache:
    """The four tensors, canaries about the codes, and what they should hold."""
    def __init__(self, rng, n_pages, H, page):
        self.codes, self.scales = _pool(rng, n_pages, H, page)
        self.d_codes = [Guarded(c.shape, torch.uint8, 0) for c in self.codes]
        for g, c in zip(self.d_codes, self.codes):
            g.t.copy_(torch.from_numpy(c))
        self.d_scales = [torch.from_numpy(s).cuda() for s in self.scales]

    def args(self):
        return [g.t.view(torch.float8_e4m3fn) for g in self.d_codes] + self.d_scales

    def check(self, what):
        for g, c, s, d in zip(self.d_codes, self.codes, self.scales, self.d_scales):
            g.check(what)
            assert np.array_equal(g.t.cpu().numpy(), c), what
            assert np.array_equal(d.cpu().numpy(), s), what


def _rows(rng, B, W, page, n_pages, live, sharing=0.5):
    """Tables and lengths of B rows, some of which begin with the whole pages of an earlier one; the pages that are left."""
    perm = list(rng.permutation(n_pages))
    table, kv = np.full((B, W), 0x7fffffff, dtype=np.int64), np.zeros(B, dtype=np.int64)
    for b in live:
        t, first = int(rng.integers(0, W * page + 1)), 0
        if b > 0 and kv[:b].max() > 0 and rng.random() < sharing:
            a = int(rng.choice(np.nonzero(kv[:b])[0]))
            first = int(rng.integers(0, min(kv[a], t) // page + 1))
            table[b, :first] = table[a, :first]
        k = ref.pages_of(t, page) - first
        if k > len(perm):
            t, k = first * page, 0
        table[b, first:first + k] = [perm.pop() for _ in range(k)]
        kv[b] = t
    return table, kv, perm


@pytest.mark.parametrize("H,page,W,B,n,short", [
    (1, 16, 1, 2, 1, False),         # one fork
    (2, 16, 9, 24, 9, False),        # ragged
    (5, 32, 40, 30, 20, True),       # the stack runs out
    (8, 64, 7, 64, 56, False),       # many of few
    (1, 128, 600, 5, 4, False),      # long rows
    (1, 16, 2, 2600, 2400, True),    # more forks than threads
])
@pytest.mark.parametrize("cut", [False, True])
def test_fork(fk, H, page, W, B, n, short, cut):
    rng = np.random.default_rng(B * 7 + W)
    n_src = B - n
    n_pages = n_src * W + n + 3
    rows = rng.permutation(B)
    table, kv, perm = _rows(rng, B, W, page, n_pages, sorted(rows[:n_src]))
    n_free = min(n // 3 if short else n, len(perm))
    free = np.full(n_pages, -9, dtype=np.int64)
    free[:n_free] = perm[:n_free]
    src, dst = rng.choice(rows[:n_src], n), rows[n_src:].copy()
    src[rng.random(n) < 0.1] = -1
    length = np.array([rng.integers(0, W * page + 9) for _ in range(n)]) if cut else None
    cache = Cache(rng, n_pages, H, page)
    want_kv, want_table, want_free, copies = share.fork(src.tolist(), dst.tolist(), None if length is None else length.tolist(), kv.tolist(),
                                                        table.tolist(), free.tolist(), n_free, page)
    for a, b, r in copies:
        for c, s in zip(cache.codes, cache.scales):
            c[b, :, :r] = c[a, :, :r]
            s[b] = s[a]
    pg = make(fk, H=H, page=page, n_pages=n_pages, W=W, B=B)
    d_table, d_kv, out = Guarded((B, W), torch.int32, 0), ref.ints(kv), Guarded((1,), torch.int32, -5)
    d_table.t.copy_(ref.ints(table))
    d_src, d_dst, d_free, d_nf = ref.ints(src), ref.ints(dst), ref.ints(free), ref.ints([n_free])
    for again in range(2):                                    # out of place the call can be repeated
        pg.fork(d_src, d_dst, d_kv, d_table.t, d_free, d_nf, out.t, *cache.args(), length=None if length is None else ref.ints(length))
    assert np.array_equal(d_kv.cpu().numpy(), want_kv) and out.t.tolist() == [want_free]
    assert np.array_equal(d_table.t.cpu().numpy(), np.asarray(want_table))
    assert np.array_equal(d_free.cpu().numpy(), free) and d_nf.tolist() == [n_free]
    cache.check("fork")
    d_table.check("table")
    out.check("n_free_out")
    assert pg.device_status() == 0
    pg.fork(d_src, d_dst, d_kv, d_table.t, d_free, d_nf, d_nf, *cache.args(), length=None if length is None else ref.ints(length))
    assert d_nf.tolist() == [want_free]
    cache.check("fork in place")


def test_fork_refuses_rows_that_cannot_be_written(fk):
    rng = np.random.default_rng(3)
    page, W, n_pages = 16, 3, 20
    pg = make(fk, page=page, n_pages=n_pages, W=W, B=6)
    cache = Cache(rng, n_pages, 2, page)
    for src, dst, ok, status in [([0, 1], [1, 3], [1], 0x106),          # a row that is a source, too
                                 ([0, 0], [0, 3], [1], 0x106),          # onto itself
                                 ([0, 1, 0], [4, 4, 5], [0, 2], 0x106),  # twice the same row: the first
                                 ([0, 6], [3, 4], [0], 0x106), ([0, 0], [3, 6], [0], 0x106), ([0, 0], [3, -1], [0], 0x106),
                                 ([-1, 0], [99, 3], [1], 0)]:           # skipped, whatever its dst
        kv, table = [20, 33, 0, 0, 0, 0], [[1, 2, 0], [3, 4, 5], [-1] * 3, [-1] * 3, [-1] * 3, [-1] * 3]
        d_kv, d_table, nf = ref.ints(kv), ref.ints(table), ref.ints([10])
        pg.fork(ref.ints(src), ref.ints(dst), d_kv, d_table, ref.ints(list(range(10, 20)) + [0] * 10), ref.ints([10]), nf, *cache.args())
        assert nf.tolist() == [10 - len(ok)], (src, dst)
        for b in range(6):
            want = [kv[src[i]] for i in ok if dst[i] == b] or [kv[b]]
            assert d_kv.tolist()[b] == want[0], (src, dst, b)
        assert pg.device_status() == status, (src, dst)
        pg.reset_device_status()


def test_fork_flags_bad_pages_lengths_and_stack(fk):
    rng = np.random.default_rng(4)
    page, W, n_pages, i = 16, 3, 20, ref.ints
    pg = make(fk, page=page, n_pages=n_pages, W=W, B=4)
    cache = Cache(rng, n_pages, 2, page)

    def go(kv, table, free, n_free, length=None):
        d_kv, nf = i(kv), i([0])
        pg.fork(i([0]), i([3]), d_kv, i(table), i(free), i([n_free]), nf, *cache.args(), length=length)
        code = pg.device_status()
        pg.reset_device_status()
        return d_kv.tolist()[3], nf.tolist()[0], code

    table, free = [[1, 2, 4]] + [[-1] * 3] * 3, list(range(20))
    assert go([20, 0, 0, 7], table, free, 6)[1:] == (5, 0)
    cache = Cache(rng, n_pages, 2, page)
    assert go([20, 0, 0, 0], [[1, 1 << 30, 4]] + [[-1] * 3] * 3, free, 6) == (20, 5, 0x101)       # the open page is not there
    assert go([20, 0, 0, 0], table, [1 << 30] * 20, 6) == (0, 5, 0x101)                           # the fresh one is not
    assert go([-5, 0, 0, 0], table, free, 6) == (0, 6, 0x103)
    assert go([48, 0, 0, 0], table, free, 6, i([-2])) == (0, 6, 0x103)
    assert go([49, 0, 0, 0], table, free, 6) == (48, 6, 0x103)                                    # cut to the table's width
    assert go([20, 0, 0, 0], table, free, -1) == (0, 0, 0x104)
    cache.check("nothing is written for any of these")
    assert go([20, 0, 0, 0], table, free, 21) == (20, 19, 0x104)
    assert go([0, 0, 0, 9], table, free, 0) == (0, 0, 0)                                          # an empty source


@pytest.mark.parametrize("page,W,B,n_pages", [(16, 4, 1, 9), (16, 30, 7, 200), (64, 9, 300, 1500), (16, 700, 5, 3000), (32, 3, 3000, 6000),
                                              (16, 2, 20000, 30000), (16, 6000, 40, 9000),
                                              (16, 200, 400, 9000), (32, 256, 256, 20000), (16, 257, 256, 20000), (64, 2, 512, 700), (64, 2, 513, 700),
                                              (16, 257, 512, 20000), (16, 3, 1024, 2000), (16, 513, 256, 20000), (16, 9, 30, 65536), (16, 9, 30, 65537)])
def test_release(fk, page, W, B, n_pages):
    rng = np.random.default_rng(B + W)
    table, kv, perm = _rows(rng, B, W, page, n_pages, range(B))
    n_new = rng.integers(-1, 3, B)
    for n_new in (n_new, np.full(B, -1), np.zeros(B, dtype=np.int64)):
        n_free = len(perm)
        free = np.full(n_pages, -9, dtype=np.int64)
        free[:n_free] = perm
        want_free, want_n, want_kv = share.release(kv.tolist(), n_new.tolist(), table.tolist(), free.tolist(), n_free, page)
        pg = make(fk, page=page, n_pages=n_pages, W=W, B=B)
        d_free, out = Guarded((n_pages,), torch.int32, 0), Guarded((B,), torch.int32, -5)
        d_free.t.copy_(ref.ints(free))
        d_t, d_n, d_table, d_nf, d_out = ref.ints(kv), ref.ints(n_new), ref.ints(table), ref.ints([n_free]), ref.ints([0])
        for again in range(2):
            pg.release(d_t, d_n, d_table, d_free.t, d_nf, out.t, d_out)
        assert np.array_equal(d_free.t.cpu().numpy(), want_free) and d_out.tolist() == [want_n]
        assert np.array_equal(out.t.cpu().numpy(), want_kv) and np.array_equal(d_t.cpu().numpy(), kv)
        d_free.check("free_pages")
        out.check("kv_len")
        pg.release(d_t, d_n, d_table, d_free.t, d_nf, d_t, d_nf)              # in place
        assert np.array_equal(d_t.cpu().numpy(), want_kv) and d_nf.tolist() == [want_n]
        assert pg.device_status() == 0


def test_release_flags_what_is_out_of_range(fk):
    pg, i = make(fk, n_pages=8, W=4, B=3), ref.ints
    table = i([[0, 1, 2, 3], [0, 4, 99, 5], [6, 7, 6, 6]])
    kv, nf = i([0] * 3), i([0])
    pg.release(i([20, 40, 64]), i([1, -1, -1]), table, i([-9] * 8), i([0]), kv, nf)
    assert kv.tolist() == [20, 0, 0] and nf.tolist() == [3] and pg.device_status() == 0x101      # 4; 6 and 7, once each
    pg.reset_device_status()
    pg.release(i([20, 32, -1]), i([1, -1, -1]), table, i([-9] * 8), i([8]), kv, nf)
    assert nf.tolist() == [8] and pg.device_status() in (0x103, 0x104)
    pg.reset_device_status()
    free = i([-9] * 8)
    pg.release(i([20, 32, 0]), i([1, -1, 0]), table, free, i([-4]), kv, nf)
    assert nf.tolist() == [1] and free.tolist() == [4] + [-9] * 7 and pg.device_status() == 0x104


@pytest.mark.parametrize("H,page,W,B,n_pages", [(1, 16, 3, 1, 5), (2, 16, 9, 6, 100), (5, 32, 20, 9, 333), (8, 64, 12, 30, 700), (3, 128, 5, 4, 31),
                                                (1, 16, 40, 300, 20000), (2, 16, 1, 3, 1),
                                                (1, 16, 50, 1500, 66000), (1, 16, 300, 4000, 65536)])
def test_compact(fk, H, page, W, B, n_pages):
    rng = np.random.default_rng(n_pages + W)
    for trial in range(3):
        table, kv, _ = _rows(rng, B, W, page, n_pages, range(B))
        if trial == 1:
            kv[:] = 0                                         # nothing in use
        if trial == 2:                                        # all in front already
            table = np.asarray(share.compact(kv.tolist(), table.tolist(), [0] * n_pages, n_pages, page)[0])
        cache = Cache(rng, n_pages, H, page)
        want_table, want_free, want_n, want_id, moves = share.compact(kv.tolist(), table.tolist(), [-9] * n_pages, n_pages, page)
        assert trial == 0 or not moves
        for x in cache.codes + cache.scales:
            for a, b in moves:
                x[b] = x[a]
        pg = make(fk, H=H, page=page, n_pages=n_pages, W=W, B=B)
        d_table, out = ref.ints(table), Guarded((B, W), torch.int32, -5)
        free, new_id, nf = Guarded((n_pages,), torch.int32, -9), Guarded((n_pages,), torch.int32, -7), ref.ints([0])
        d_kv = ref.ints(kv)
        for again in range(2):
            pg.compact(d_kv, d_table, out.t, free.t, nf, new_id.t, *cache.args())
        for name, g, want in (("table", out, want_table), ("free", free, want_free), ("new_id", new_id, want_id)):
            assert np.array_equal(g.t.cpu().numpy(), np.asarray(want).reshape(g.t.shape)), (name, trial)
            g.check(name)
        assert nf.tolist() == [want_n] and np.array_equal(d_table.cpu().numpy(), table)
        cache.check("compact")
        pg.compact(d_kv, d_table, d_table, free.t, nf, new_id.t, *cache.args())      # in place
        assert np.array_equal(d_table.cpu().numpy(), np.asarray(want_table))
        assert pg.device_status() == 0


def test_compact_flags_pages_outside_the_pool(fk):
    rng = np.random.default_rng(5)
    pg, i = make(fk, n_pages=8, W=3, B=2), ref.ints
    cache = Cache(rng, 8, 2, 16)
    table, nf, new_id, free = i([[7, -3, 2], [8, 5, 5]]), i([0]), i([0] * 8), i([0] * 8)
    pg.compact(i([48, 30]), table, table, free, nf, new_id, *cache.args())
    assert table.tolist() == [[1, -3, 2], [8, 0, 5]] and nf.tolist() == [5] and pg.device_status() == 0x101
    assert new_id.tolist() == [-1, -1, 2, -1, -1, 0, -1, 1] and free.tolist()[:5] == [7, 6, 5, 4, 3]
    pg.reset_device_status()
    pg.compact(i([-1, 1000]), table, table, free, nf, new_id, *cache.args())
    assert pg.device_status() in (0x101, 0x103)


@pytest.mark.parametrize("capture", [False, True])
def test_shared_pages_on_another_stream_and_captured(fk, capture):
    """fork, release and compact on a side stream behind a slow one, or captured and replayed twice."""
    rng = np.random.default_rng(8)
    page, W, B, n_pages = 16, 6, 6, 60
    table, kv, perm = _rows(rng, B, W, page, n_pages, [0, 1])
    kv[0] = 37
    table[0, :3] = [perm.pop() for _ in range(3)]
    free = np.asarray(perm + [-1] * (n_pages - len(perm)))
    pg, cache = make(fk, page=page, n_pages=n_pages, W=W, B=B), Cache(rng, n_pages, 2, page)
    src, dst, n_new = [0, 1, 0], [2, 3, 4], [1, -1, 1, 1, -1, 0]
    kv1, table1, nf1, copies = share.fork(src, dst, None, kv.tolist(), table.tolist(), free.tolist(), len(perm), page)
    free2, nf2, kv2 = share.release(kv1, n_new, table1, free.tolist(), nf1, page)
    table3, free3, nf3, _, moves = share.compact(kv2, table1, free2, n_pages, page)
    for x, is_code in [(c, True) for c in cache.codes] + [(s, False) for s in cache.scales]:
        for a, b, r in copies:
            if is_code:
                x[b, :, :r] = x[a, :, :r]
            else:
                x[b] = x[a]
        for a, b in moves:
            x[b] = x[a]
    base = [ref.ints(x) for x in (kv, table, free, [len(perm)])]
    d_kv, d_table, d_free, d_nf = [x.clone() for x in base]
    start = [x.clone() for x in cache.args()[2:]] + [g.t.clone() for g in cache.d_codes]
    d_src, d_dst, d_new, new_id = ref.ints(src), ref.ints(dst), ref.ints(n_new), ref.ints([0] * n_pages)

    def life():
        for x, y in zip((d_kv, d_table, d_free, d_nf, *cache.d_scales, *[g.t for g in cache.d_codes]), (*base, *start)):
            x.copy_(y)
        pg.fork(d_src, d_dst, d_kv, d_table, d_free, d_nf, d_nf, *cache.args())
        pg.release(d_kv, d_new, d_table, d_free, d_nf, d_kv, d_nf)
        pg.compact(d_kv, d_table, d_table, d_free, d_nf, new_id, *cache.args())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        if capture:
            life()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                life()
            graph.replay()
            graph.replay()
        else:
            torch.cuda._sleep(20_000_000)
            life()
    side.synchronize()
    assert d_kv.tolist() == kv2 and d_nf.tolist() == [nf3]
    assert np.array_equal(d_table.cpu().numpy(), np.asarray(table3)) and np.array_equal(d_free.cpu().numpy(), free3)
    cache.check("life")
    assert pg.device_status() == 0


def test_requests_that_share_pages_live_and_end(fk):
    """Sixty steps of a small server: requests begin, fork, take tokens, finish, the pool is compacted; rows read back equal what each
    request was given, and every page is in one place."""
    rng = np.random.default_rng(11)
    H, page, W, B, n_pages = 2, 16, 8, 10, 90
    pg = make(fk, H=H, page=page, n_pages=n_pages, W=W, B=B, dtype=torch.float32)
    k_pages, v_pages, k_scale, v_scale = cache = pg.alloc()
    for x in cache[:2]:
        x.view(torch.uint8).fill_(0)
    d_kv, d_table, d_free, d_nf = ref.ints([0] * B), ref.ints(np.full((B, W), -1)), ref.ints(range(n_pages)), ref.ints([n_pages])
    q_start, new_id = ref.ints([0] * (B + 1)), ref.ints([0] * n_pages)
    rows = [np.zeros((0, H, 128)) for _ in range(B)]
    for step in range(60):
        busy = [b for b in range(B) if len(rows[b])]
        idle = [b for b in range(B) if not len(rows[b])]
        if busy and idle and step % 3 == 0:
            dst = list(rng.permutation(idle)[:rng.integers(1, len(idle) + 1)])
            src = [int(rng.choice(busy)) for _ in dst]
            length = [int(rng.integers(1, len(rows[s]) + 1)) for s in src]
            pg.fork(ref.ints(src), ref.ints(dst), d_kv, d_table, d_free, d_nf, d_nf, *cache, length=ref.ints(length))
            for s, d, n in zip(src, dst, length):
                rows[d] = rows[s][:n].copy()
        n_new = rng.integers(0, 12, B)
        for b in range(B):
            if len(rows[b]) and (rng.random() < 0.2 or len(rows[b]) + n_new[b] > W * page):
                n_new[b] = -1
        d_new = ref.ints(n_new)
        pg.release(d_kv, d_new, d_table, d_free, d_nf, d_kv, d_nf)
        total = int(np.maximum(n_new, 0).sum())
        slots = ref.ints([0] * total)
        pg.tables(d_kv, d_new, d_table, d_free, d_nf, q_start, d_kv, slots, d_nf)
        x = rng.standard_normal((total, H, 128))
        x = ref.VALUES[ref.encode(x * 100)] / 128             # exact in the cache unless a page's scale has to grow
        x[:, :, 0] = 3.5                                      # which this keeps from happening: every row has the same largest element
        new = torch.from_numpy(x).float().cuda()
        pg.store(new, new, slots, *cache)
        at = 0
        for b in range(B):
            if n_new[b] < 0:
                rows[b] = rows[b][:0]
            else:
                rows[b] = np.concatenate([rows[b], x[at:at + n_new[b]]])
                at += n_new[b]
        if step % 7 == 6:
            pg.compact(d_kv, d_table, d_table, d_free, d_nf, new_id, *cache)
        assert d_kv.tolist() == [len(r) for r in rows], step
        L = max(1, max(len(r) for r in rows))
        K, V = pg.load(d_kv, d_table, *cache, L)
        for b in range(B):
            want = np.zeros((L, H, 128))
            want[:len(rows[b])] = rows[b]
            assert np.array_equal(K[b].cpu().numpy(), want.transpose(1, 0, 2)) and torch.equal(K[b], V[b]), (step, b)
        named = {p for r, row in zip(rows, d_table.tolist()) for p in row[:ref.pages_of(len(r), page)]}
        free = d_free.tolist()[:d_nf.item()]
        assert len(set(free)) == len(free) and named | set(free) == set(range(n_pages)) and not named & set(free), step
    assert pg.device_status() == 0


def test_the_c_calls_refuse_what_they_cannot_do(fk):
    """NULL and misaligned tensors, counts outside the handle's: an error code and a text, and nothing is launched."""
    rng = np.random.default_rng(1)
    pg = make(fk, n_pages=6, W=3, B=4)
    big = make(fk, n_pages=6, W=1 << 26, B=40)
    cache = Cache(rng, 6, 2, 16)
    i = ref.ints([0] * 64).data_ptr()
    c = [x.data_ptr() for x in cache.args()]
    lib, n0 = fk.load(), pg.launch_count()
    fork, release, compact = lib.faedkv_pages_fork, lib.faedkv_pages_release, lib.faedkv_pages_compact
    # arguments, where the batch stands, which others are no tensors, which may be NULL (fork: the lengths, and a workspace that few forks do not need)
    calls = [(fork, [pg._h, i, i, i, 4, 4, i, i, i, i, i, *c, i, None], 5, (4,), (3, 15)), (release, [pg._h, i, i, 4, i, i, i, i, i, i, None], 3, (), ()),
             (compact, [pg._h, i, 4, i, i, i, i, i, *c, i, None], 2, (), ())]
    for call, good, at, counts, optional in calls:
        for k, x in enumerate(good[1:-1], 1):
            if k == at or k in counts:
                continue
            if k not in optional:
                assert call(*good[:k], None, *good[k + 1:]) == -1, (call.__name__, k)
            assert call(*good[:k], x + 2, *good[k + 1:]) == -5, (call.__name__, k)
            assert b"aligned" in lib.faedkv_pages_last_error(pg._h)
        for batch in (0, -1, 5):
            assert call(*good[:at], batch, *good[at + 1:]) == -3, (call.__name__, batch)
        assert call(big._h, *good[1:at], 32, *good[at + 1:]) == -3
        assert b"2^31" in lib.faedkv_pages_last_error(big._h)
    good = calls[0][1]
    for n in (-1, 5):
        assert fork(*good[:4], n, *good[5:]) == -3
        assert lib.faedkv_pages_fork_bytes(pg._h, 4, n) == 0
    many = make(fk, n_pages=6, W=3, B=5000)
    assert lib.faedkv_pages_fork_bytes(pg._h, 4, 4) == 0 and lib.faedkv_pages_fork_bytes(many._h, 5000, 4) == 4 * 5004
    assert fork(many._h, *good[1:5], 5000, *good[6:15], None, None) == -1 and many.launch_count() == 0
    assert pg.launch_count() == n0 and big.launch_count() == 0 and pg.device_status() == 0
    out = ref.ints([0])
    pg.fork(ref.ints([]), ref.ints([]), ref.ints([0] * 4), ref.ints(np.zeros((4, 3))), ref.ints([0] * 6), ref.ints([5]), out, *cache.args())
    assert out.tolist() == [5]                                # no forks: the height is passed on
    cache.check("refused")
