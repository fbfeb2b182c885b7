"""The form with query columns as rows where its branches are rarely taken: NaN and pages that are not there, captured prompts, two calls at once; and the
form with eight columns at its own, narrower bound."""
import math

import numpy as np
import pytest
import torch

import pages_ref as ref
from attn_bounds import attention, close
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


def rows_left(args, names, b, n, page, gone):
    """K, V of row b without the tokens of its pages `gone`, in 64 bits, [H, tokens, 128] each."""
    a = dict(zip(names, args))
    keep = [t for t in range(n) if t // page not in gone]
    row = [p if 0 <= p < a["k_pages"].shape[0] else 0 for p in a["table"][b].tolist()[:ref.pages_of(n, page)]]
    return [torch.from_numpy(ref.rows_of(c.view(torch.uint8).cpu().numpy(), s.double().cpu().numpy(), row, n, page)).cuda()[:, keep]
            for c, s in ((a["k_pages"], a["k_scale"]), (a["v_pages"], a["v_scale"]))], keep


SHARED = ("q", "kv_len", "table", "group_start", "shared_len", "k_pages", "v_pages", "k_scale", "v_scale", "out")
DIFF = ("q", "kv_len", "table", "k_pages", "v_pages", "k_scale", "v_scale", "lam", "out")


@pytest.mark.parametrize("page,G,shared,rows", [(16, 8, 640, 40), (64, 2, 1280, 50), (128, 4, 2560, 64), (32, 1, 96, 33)])
def test_shared_nan(fk, page, G, shared, rows):
    """In a shared page a NaN value reaches its channel of every row, a NaN key every channel; behind it, the row that holds it."""
    lens = [shared + 1 + 7 * i % 40 for i in range(rows)]

    def value(table, kc, vc):
        vc[table[0][1], 0, 5, 9] = 127
        vc[table[rows - 1][shared // page], 0, 0, 77] = 255

    def key(table, kc, vc):
        kc[table[3][shared // page], 0, 0, 5] = 127

    _, _, out = shared_case(fk, torch.bfloat16, page, 1, G, [(shared, lens)], edit=value, check_rows=[], width=100000)
    want = torch.zeros_like(out, dtype=torch.bool)
    want[:, :, 9] = True
    want[rows - 1, :, 77] = True
    assert torch.equal(torch.isnan(out), want)
    _, _, out = shared_case(fk, torch.bfloat16, page, 1, G, [(shared, lens)], edit=key, check_rows=[], width=100000)
    want.zero_()
    want[3] = True
    assert torch.equal(torch.isnan(out), want)

    def shared_key(table, kc, vc):
        kc[table[0][0], 0, 2, 5] = 127

    _, _, out = shared_case(fk, torch.bfloat16, page, 1, G, [(shared, lens)], edit=shared_key, check_rows=[], width=100000)
    assert bool(torch.isnan(out).all())


@pytest.mark.parametrize("page,G,shared,rows", [(16, 8, 640, 40), (64, 2, 1280, 50), (128, 4, 384, 64), (32, 1, 96, 33)])
@pytest.mark.parametrize("bad", [-5, 0x7fffffff])
def test_shared_pages_that_are_not_there(fk, page, G, shared, rows, bad):
    """They count as no tokens: one in the middle, the first, a whole tile of them; all that a group shares."""
    whole = shared // page
    for gone in ({whole // 2}, {0}, set(range(max(0, whole - 128 // page), whole)), set(range(whole))):
        def missing(table, kc, vc):
            for p in gone:
                table[:, p] = bad

        lens = [shared + 1 + 7 * i % 40 for i in range(rows)]
        pg, args, out = shared_case(fk, torch.bfloat16, page, 1, G, [(shared, lens)], edit=missing, check_rows=[], status=0x101, width=100000)
        for b in (0, 1, rows // 2, rows - 1):
            (K, V), keep = rows_left(args, SHARED, b, lens[b], page, gone)
            want, tol = attention("wide", args[0][b], K[0], V[0], torch.full((G,), len(keep), device="cuda"), 1 / math.sqrt(128))
            close(out[b], want, tol, (b, gone))


@pytest.mark.parametrize("page,G,n,new,gone", [(16, 4, 900, 70, {3}), (16, 2, 300, 290, {0, 5}), (64, 1, 1500, 200, {0, 1, 2, 3}), (128, 4, 500, 40, {1}),
                                               (32, 2, 256, 100, {4, 5, 6, 7}), (16, 1, 40, 30, {0, 1, 2})])
@pytest.mark.parametrize("dtype,width", [(torch.bfloat16, 60000), (torch.bfloat16, 1), (torch.float32, 1)])
def test_differential_prompts_over_pages_that_are_not_there(fk, dtype, width, page, G, n, new, gone):
    pg, args, kw, out = diff_case(fk, dtype, page, 1, G, [n], [new], gain=False, width=width)
    a = dict(zip(DIFF, args))
    for p in gone:
        a["table"][0, p] = -7
    pg.attn_diff(*args, **kw)
    assert pg.device_status() == 0x101
    (K, V), keep = rows_left(args, DIFF, 0, n, page, gone)
    seen = torch.tensor([sum(t < n - new + 1 + i for t in keep) for i in range(new)], device="cuda")
    expect(out, "f32" if dtype == torch.float32 else "wide", a["q"], K[0], V[0], seen, 0.125, a["lam"], None, 0.0, gone)


@pytest.mark.parametrize("lens,new", [([5000], [40]), ([700, 300], [100, 20]), ([3000, 129, 64], [10, 129, 33])])
@pytest.mark.parametrize("gain", [True, False])
def test_captured_differential_prompts(fk, lens, new, gain):
    """Two graphs on one workspace, replayed one after the other, on another stream and with other queries."""
    pg, args, kw, out = diff_case(fk, torch.bfloat16, 64, 2, 4, lens, new, gain=gain, width=60000)
    want, q0 = out.clone(), args[0].clone()
    ws = torch.empty(pg.attn_diff_bytes(len(lens), sum(new)), dtype=torch.uint8, device="cuda")
    args[0].mul_(-0.5)
    pg.attn_diff(*args, **kw)
    other, q1 = out.clone(), args[0].clone()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            pg.attn_diff(*args, **kw, ws=ws)
        graphs.append(graph)
    side = torch.cuda.Stream()
    for i in range(6):
        with torch.cuda.stream(side):
            out.zero_()
            ws.fill_(255)
            args[0].copy_(q1 if i & 2 else q0)
            graphs[i & 1].replay()
        side.synchronize()
        assert torch.equal(out, other if i & 2 else want)
    assert pg.device_status() == 0


def test_differential_prompts_beside_other_calls(fk):
    """Prompts, a decode step over shared pages and one of differential heads on streams of their own: again and again, the same bits."""
    calls = []
    for lens, new in (([4000, 700], [60, 200]), ([9000], [130])):
        pg, args, kw, out = diff_case(fk, torch.bfloat16, 32, 2, 4, lens, new, width=60000)
        ws = torch.empty(pg.attn_diff_bytes(len(lens), sum(new)), dtype=torch.uint8, device="cuda")
        calls.append((pg, lambda pg=pg, args=args, kw=kw, ws=ws: pg.attn_diff(*args, **kw, ws=ws), out, out.clone()))
    pg, args, kw, out = diff_case(fk, torch.bfloat16, 64, 2, 4, [4000, 90, 700])
    ws = torch.empty(pg.attn_diff_bytes(3, 3), dtype=torch.uint8, device="cuda")
    calls.append((pg, lambda pg=pg, args=args, kw=kw, ws=ws: pg.attn_diff(*args, **kw, ws=ws), out, out.clone()))
    pg, args, out = shared_case(fk, torch.bfloat16, 16, 2, 4, [(2048, [2050 + 7 * i for i in range(70)])], width=50000)
    ws = torch.empty(pg.attn_shared_bytes(70, 1), dtype=torch.uint8, device="cuda")
    calls.append((pg, lambda pg=pg, args=args, ws=ws: pg.attn_shared(*args, ws=ws), out, out.clone()))
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(8):
        torch.cuda.synchronize()
        for _ in range(3):
            for (pg, call, out, want), stream in zip(calls, streams):
                with torch.cuda.stream(stream):
                    out.zero_()
                    call()
        torch.cuda.synchronize()
        for pg, call, out, want in calls:
            assert torch.equal(out, want) and pg.device_status() == 0


@pytest.mark.parametrize("page,H,G,groups", [
    (16, 2, 4, [(128, [128, 129, 128, 200, 131])]), (64, 3, 3, [(0, [40, 1, 0]), (640, [641, 700, 900]), (64, [65])]),
    (128, 2, 8, [(256, [300, 256]), (128, [1000, 129, 128, 500])]), (64, 8, 5, [(1280, [1281] * 9), (1280, [1400] * 3)]),
])
def test_eight_columns_hold_their_own_bound(fk, page, H, G, groups):
    """Tables of few pages take eight columns a block, with weights to 2^-12 and 2^-34 as a decode step of attn() has them."""
    pg, args, out = shared_case(fk, torch.bfloat16, page, H, G, groups, check_rows=[])
    for b, n in enumerate(args[1].tolist()):
        (K, V), _ = rows_left(args, SHARED, b, n, page, ())
        for h in range(H):
            hs = slice(h * G, (h + 1) * G)
            close(out[b, hs], *attention("bf16", args[0][b, hs], K[h], V[h], torch.full((G,), n, device="cuda"), 1 / math.sqrt(128)), (b, h))
