"""A decode step over pages that rows share, on the GPU against softmax attention of each row in 64 bits."""
import math

import numpy as np
import pytest
import torch

import pages_ref as ref
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


def layout(rng, page, groups):
    """groups: (tokens shared, lengths of the rows).  Rows name their group's pages as far as they reach and pages of their own behind;
    what lies behind a row's end is no page."""
    n_pages = sum(s // page + sum(max(0, ref.pages_of(n, page) - s // page) for n in lens) for s, lens in groups) + 2
    perm = list(rng.permutation(n_pages))
    W = max([ref.pages_of(n, page) for _, lens in groups for n in lens] + [s // page for s, _ in groups] + [1]) + 1
    table, lens = [], []
    for s, rows in groups:
        common = [perm.pop() for _ in range(s // page)]
        for n in rows:
            k = ref.pages_of(n, page)
            row = common[:k]
            row += [perm.pop() for _ in range(k - len(row))]
            table.append(row + [0x7fffffff] * (W - k))
            lens.append(n)
    return np.asarray(table), lens, n_pages, W


def case(fk, dtype, page, H, G, groups, shared=None, starts=None, status=0, scale=None, qmul=1.0, pow2=True, strided=False, edit=None, check_rows=None, width=0):
    rng = np.random.default_rng(sum(s for s, _ in groups) + page + 31 * H + G)
    table, lens, n_pages, W = layout(rng, page, groups)
    B = len(lens)
    if width:                                                # wide tables: bf16 groups of many query columns take the form with rows
        table = np.concatenate([table, np.full((B, width), 0x7fffffff)], axis=1)
        W += width
    (kc, ks), (vc, vs) = [ref.random_cache(rng, n_pages, H, page, lens, table, pow2) for _ in range(2)]
    if edit is not None:
        edit(table, kc, vc)
    pg = fk.Pages(n_kv_heads=H, n_q_heads=H * G, page_size=page, n_pages=n_pages, max_pages=W, max_batch=B,
                  kv_dtype=fk.BF16 if dtype == torch.bfloat16 else fk.F32)
    wide = torch.from_numpy(rng.standard_normal((B, 3 * H * G, 128)) * qmul).to(dtype).cuda()
    q = wide[:, H * G:2 * H * G] if strided else wide[:, :H * G].contiguous()
    out = torch.full((B, H * G, 128), 7.0, dtype=dtype, device="cuda")
    starts = np.concatenate([[0], np.cumsum([len(r) for _, r in groups])]) if starts is None else starts
    shared = [s for s, _ in groups] if shared is None else shared
    args = (q, ref.ints(lens), ref.ints(table), ref.ints(starts), ref.ints(shared), ref.cuda8(kc), ref.cuda8(vc), ref.cuda32(ks), ref.cuda32(vs),
            out)
    pg.attn_shared(*args, scale=scale or 0.0)
    kind = "f32" if dtype == torch.float32 else "wide"
    for b in range(B) if check_rows is None else check_rows:
        K, V = [torch.from_numpy(ref.rows_of(c, s, table[b], lens[b], page)).cuda() for c, s in ((kc, ks), (vc, vs))]
        for h in range(H):
            hs = slice(h * G, (h + 1) * G)
            want, tol = attention(kind, q[b, hs], K[h], V[h], torch.full((G,), lens[b], device="cuda"), scale or 1 / math.sqrt(128))
            close(out[b, hs], want, tol, (b, h))
    assert pg.device_status() == status
    pg.reset_device_status()
    return pg, args, out


BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])


@BOTH
@pytest.mark.parametrize("page,H,G,groups", [
    (16, 1, 1, [(16, [17, 30])]),                                          # the smallest group
    (16, 2, 4, [(128, [128, 129, 128, 200, 131])]),                        # some rows end where the shared tokens do
    (64, 3, 3, [(0, [40, 1, 0]), (640, [641, 700, 900]), (64, [65])]),     # nothing shared; a group of one
    (32, 1, 7, [(960, [1000] * 11), (0, [77]), (32, [33, 64])]),           # more rows than a block takes
    (128, 2, 8, [(256, [300, 256]), (128, [1000, 129, 128, 500])]),
    (16, 4, 2, [(2000, [2001 + 7 * i for i in range(40)])]),               # split over CTAs; tails split from it
    (64, 8, 5, [(1280, [1281] * 9), (1280, [1400] * 3)]),
    (32, 2, 6, [(96, [100, 97]), (96, [100, 97, 99]), (192, [200, 201, 202, 203])]),
    (16, 1, 8, [(48, [50] * 33)]),
])
def test_groups(fk, dtype, page, H, G, groups):
    case(fk, dtype, page, H, G, groups, pow2=page != 32, strided=page == 64)
    if dtype == torch.bfloat16:
        case(fk, dtype, page, H, G, groups, pow2=page != 32, width=100000, qmul=3.0 if page == 128 else 1.0)


@pytest.mark.parametrize("page,H,G,groups", [
    (16, 1, 8, [(2048, [2050] * 33)]),                                     # two row tiles and some, split over CTAs
    (64, 2, 4, [(4096, [4100 + 9 * i for i in range(64)]), (640, [700] * 12)]),
    (32, 5, 2, [(1600, [1601 + i for i in range(64)])]),                   # one row tile of 128
    (16, 2, 7, [(160, [0, 150, 161, 160, 17, 300] + [170] * 31)]),         # rows shorter than their group among many
    (128, 1, 5, [(8192, [8200] * 13), (0, [5] * 13)]),
])
def test_groups_of_many_columns(fk, page, H, G, groups):
    case(fk, torch.bfloat16, page, H, G, groups, width=50000)
    case(fk, torch.bfloat16, page, H, G, groups, width=50000, qmul=5.0, strided=True, pow2=False)


@BOTH
def test_rows_shorter_than_their_group(fk, dtype):
    """A row that holds less than its group shares is attended alone: an empty one, a short one, the first of its block; rows of a
    block of which none has them all."""
    case(fk, dtype, 16, 2, 4, [(160, [0, 150, 161, 160, 17, 300])])
    case(fk, dtype, 16, 2, 4, [(160, [159, 1, 0, 33])])
    case(fk, dtype, 16, 1, 8, [(320, [5] * 20 + [400] * 3 + [0] * 9 + [321, 320])])


@BOTH
def test_shared_lengths_that_are_not_whole_pages(fk, dtype):
    case(fk, dtype, 32, 2, 2, [(320, [330, 350, 321])], shared=[319])
    case(fk, dtype, 32, 2, 2, [(320, [330, 350, 321]), (64, [70, 90])], shared=[31, 65])
    case(fk, dtype, 32, 2, 2, [(320, [330, 350, 321])], shared=[0])


@BOTH
def test_empty_groups_and_rows_of_no_group(fk, dtype):
    g = [(64, [70, 80]), (128, [130, 140, 150])]
    case(fk, dtype, 16, 2, 4, g, starts=[0, 0, 2, 2, 5], shared=[64, 64, 0, 128])
    case(fk, dtype, 16, 2, 4, g, starts=[0, 2], shared=[64], status=0x105)                 # the last three rows are in none
    case(fk, dtype, 16, 2, 4, g, starts=[1, 2, 5], shared=[999, 128], status=0x105)        # nor is the first
    case(fk, dtype, 16, 2, 4, g, starts=[0, 2, 9], shared=[64, 128], status=0x105)         # ends behind the batch
    case(fk, dtype, 16, 2, 4, g, starts=[-3, 2, 5], shared=[64, 128], status=0x105)
    case(fk, dtype, 16, 2, 4, g, shared=[64, -16], status=0x103)
    case(fk, dtype, 16, 2, 4, g, shared=[1 << 30, 128], status=0x103)


@BOTH
def test_more_blocks_than_are_shared_out(fk, dtype):
    rng = np.random.default_rng(4)
    groups = []
    for _ in range(160):
        s = int(rng.integers(0, 5)) * 16
        groups.append((s, [s + int(rng.integers(0, 40)) for _ in range(rng.integers(1, 12))]))
    groups.append((48, [60 + i % 9 for i in range(300)]))
    assert sum(len(r) for _, r in groups) > 1024
    rows = sum(len(r) for _, r in groups)
    case(fk, dtype, 16, 2, 2, groups, check_rows=sorted({*range(0, rows, 5), *range(rows - 40, rows)}))
    if dtype == torch.bfloat16:
        groups = [(96, [100 + i % 30 for i in range(700)]), (32, [33] * 400 + [50] * 20)]
        case(fk, dtype, 16, 1, 2, groups, check_rows=range(0, 1120, 9), width=5000)


@BOTH
def test_scale_and_sharp_scores(fk, dtype):
    case(fk, dtype, 16, 2, 4, [(300 // 16 * 16, [300, 310, 333])], scale=0.3)
    case(fk, dtype, 64, 1, 4, [(1280, [1300] * 5)], qmul=8.0)              # one token takes nearly all: in the shared part, or behind it


@BOTH
def test_nan_and_missing_pages(fk, dtype):
    """A NaN value in a shared page reaches its channel of every row; one behind the shared tokens only the row that holds it.  A
    page that is not there counts as no tokens."""
    groups = [(64, [70, 64, 90])]

    def nan(table, kc, vc):
        vc[table[0][2], 0, 5, 9] = 127
        vc[table[2][4], 0, 3, 77] = 255

    pg, args, out = case(fk, dtype, 16, 1, 2, groups, edit=nan, check_rows=[])
    want = torch.zeros_like(out, dtype=torch.bool)
    want[:, :, 9] = True
    want[2, :, 77] = True
    assert torch.equal(torch.isnan(out), want)

    def missing(table, kc, vc):
        table[0][1] = table[1][1] = table[2][1] = -5

    rng = np.random.default_rng(0)
    pg, args, out = case(fk, dtype, 16, 1, 2, groups, edit=missing, check_rows=[], status=0x101)
    q, kv, table, _, _, kp, vp, ks, vs, _ = args
    for b, n in enumerate([70, 64, 90]):
        keep = [t for t in range(n) if t // 16 != 1]
        row = [p if 0 <= p < kp.shape[0] else 0 for p in table[b].tolist()]
        K, V = [torch.from_numpy(ref.rows_of(c.view(torch.uint8).cpu().numpy(), s.double().cpu().numpy(), row, n, 16)).cuda()[0, keep]
                for c, s in ((kp, ks), (vp, vs))]
        want, tol = attention("f32" if dtype == torch.float32 else "wide", q[b], K, V, torch.full((2,), len(keep), device="cuda"), 1 / math.sqrt(128))
        close(out[b], want, tol, b)


def test_a_call_gives_the_same_bits_again(fk):
    pg, args, out = case(fk, torch.bfloat16, 64, 2, 4, [(6400, [6400 + 3 * i for i in range(24)])])
    first = out.clone()
    for _ in range(5):
        out.zero_()
        pg.attn_shared(*args)
        assert torch.equal(out, first)


@pytest.mark.parametrize("groups", [
    [(20480, [20500 + i for i in range(64)]), (30848, [30900] * 20)],        # a block of 80 columns behind one of 256, on one CTA
    [(20480, [20500 + i for i in range(70)])],
])
def test_many_columns_give_the_same_bits_again(fk, groups):
    pg, args, out = case(fk, torch.bfloat16, 64, 2, 4, groups, width=50000)
    first = out.clone()
    for _ in range(10):
        out.zero_()
        pg.attn_shared(*args)
        assert torch.equal(out, first)


def test_captured_and_on_another_stream(fk):
    pg, args, out = case(fk, torch.bfloat16, 64, 2, 4, [(640, [700, 641, 999]), (0, [5, 130])])
    want, q0 = out.clone(), args[0].clone()
    args[0].zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        args[0].copy_(q0)
        pg.attn_shared(*args)
    side.synchronize()
    assert torch.equal(out, want)
    ws = torch.empty(pg.attn_shared_bytes(5, 2), dtype=torch.uint8, device="cuda")
    graphs = []
    for _ in range(2):                                         # two graphs on one workspace, replayed one after the other
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            pg.attn_shared(*args, ws=ws)
        graphs.append(graph)
    for i in range(4):
        out.zero_()
        ws.fill_(255)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_two_calls_at_once(fk):
    """Two streams with a workspace each, launches of both forms side by side: again and again, the same bits."""
    pairs = []
    for groups in ([(2048, [2050 + 7 * i for i in range(70)]), (640, [700] * 9)], [(4096, [4200] * 33)]):
        pg, args, out = case(fk, torch.bfloat16, 16, 2, 4, groups, width=50000)
        n = len(args[1])
        ws = torch.empty(pg.attn_shared_bytes(n, len(groups)), dtype=torch.uint8, device="cuda")
        pairs.append((pg, args, out, out.clone(), ws, torch.cuda.Stream()))
    for _ in range(5):
        torch.cuda.synchronize()
        for pg, args, out, want, ws, st in pairs:
            with torch.cuda.stream(st):
                for _ in range(3):
                    out.zero_()
                    pg.attn_shared(*args, ws=ws)
        torch.cuda.synchronize()
        for pg, args, out, want, ws, st in pairs:
            assert torch.equal(out, want) and pg.device_status() == 0


def test_lengths_that_grow_under_a_captured_step(fk):
    """The lengths are read on the device: a graph of one step serves rows as they grow past their shared tokens."""
    rng = np.random.default_rng(9)
    page, groups = 16, [(64, [80, 80, 80])]
    pg, args, out = case(fk, torch.bfloat16, page, 1, 4, groups)
    q, kv, table, _, _, kp, vp, ks, vs, _ = args
    ws = torch.empty(pg.attn_shared_bytes(3, 1), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pg.attn_shared(*args, ws=ws)
    for lens in ([64, 65, 80], [10, 64, 70], [80, 1, 0], [80, 80, 80]):
        kv.copy_(ref.ints(lens))
        graph.replay()
        for b, n in enumerate(lens):
            K, V = [torch.from_numpy(ref.rows_of(c.view(torch.uint8).cpu().numpy(), s.double().cpu().numpy(), table[b].tolist(), n, page)).cuda()
                    for c, s in ((kp, ks), (vp, vs))]
            want, tol = attention("wide", q[b], K[0], V[0], torch.full((4,), n, device="cuda"), 1 / math.sqrt(128))
            close(out[b], want, tol, (lens, b))


def test_refusals(fk):
    pg, args, out = case(fk, torch.bfloat16, 16, 2, 2, [(16, [33, 20])])
    lib, z, n0 = fk.load(), None, pg.launch_count()
    p = [x.data_ptr() for x in args]
    ws = torch.empty(pg.attn_shared_bytes(2, 1), dtype=torch.uint8, device="cuda")
    good = [pg._h, p[0], 512, p[3], p[4], 1, 2, p[1], p[2], p[5], p[6], p[7], p[8], 0.0, p[9], ws.data_ptr(), ws.numel(), z]
    for k in (1, 3, 4, 7, 8, 9, 10, 11, 12, 14, 15):
        assert lib.faedkv_pages_attn_shared(*good[:k], z, *good[k + 1:]) == -1, k
        assert lib.faedkv_pages_attn_shared(*good[:k], good[k] + 2, *good[k + 1:]) == -5, k
    for k, bad, code in [(2, 511, -3), (2, 515, -5), (5, 0, -3), (5, 3, -3), (6, 0, -3), (6, 3, -3), (13, -1.0, -1), (13, math.inf, -1), (13, math.nan, -1),
                         (16, ws.numel() - 1, -3)]:
        assert lib.faedkv_pages_attn_shared(*good[:k], bad, *good[k + 1:]) == code, (k, bad)
    names = ("q", "kv_len", "table", "group_start", "shared_len", "k_pages", "v_pages", "k_scale", "v_scale", "out")
    a = dict(zip(names, args))
    for name, bad in (("q", a["q"][:1]), ("q", a["q"].float()), ("group_start", a["group_start"][:1]), ("shared_len", a["shared_len"].long()),
                      ("out", out[:1]), ("table", a["table"][:, :1])):
        with pytest.raises(ValueError, match=name):
            pg.attn_shared(**{**a, name: bad})
    assert pg.launch_count() == n0
