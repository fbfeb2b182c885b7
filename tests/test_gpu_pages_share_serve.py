"""Answers to shared prompts from their first token to their last: the calls on shared pages, store, tables and both attentions together."""
import math

import numpy as np
import pytest
import torch

import pages_ref as ref
from attn_bounds import attention, close
from test_gpu_pages_diff import expect

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fk():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2507_20030_b200 import binding, build
    build.build()
    binding.load()
    return binding


@pytest.mark.parametrize("dtype,page,H,G,width,answers", [
    (torch.bfloat16, 16, 2, 4, 0, (5, 3)),
    (torch.float32, 32, 1, 3, 0, (2, 6)),
    (torch.bfloat16, 64, 2, 4, 50000, (70, 4)),              # wide tables: the form with rows for the groups
])
def test_answers_to_shared_prompts(fk, dtype, page, H, G, width, answers):
    """Two prompts are stored, forked into their answers, decoded by a captured step (tables, store, both attentions), one answer of each
    ends, the pool is compacted, and the decoding goes on: every output against 64 bits over the rows that the cache holds."""
    rng = np.random.default_rng(page + H + G)
    prompts, HQ = (5 * page + 3, 9 * page), H * G
    B, W = 2 + sum(answers), 14 + width
    n_pages = 14 * 2 + 4 * B
    pg = fk.Pages(n_kv_heads=H, n_q_heads=HQ, page_size=page, n_pages=n_pages, max_pages=W, max_batch=B,
                  kv_dtype=fk.BF16 if dtype == torch.bfloat16 else fk.F32)
    cache, i = pg.alloc(), ref.ints
    kv, nf, q_start = i([0] * B), i([n_pages]), i([0] * (B + 1))
    table, free, new_id = i(np.full((B, W), -1)), i(np.arange(n_pages)), i([0] * n_pages)
    # the prompts in the first row of each group
    bounds = [0, 1 + answers[0], B]
    n_new = np.zeros(B, int)
    n_new[bounds[0]], n_new[bounds[1]] = prompts
    slots = i([0] * sum(prompts))
    pg.tables(kv, i(n_new), table, free, nf, q_start, kv, slots, nf)

    def rows(n, heads):
        return torch.from_numpy(rng.standard_normal((n, heads, 128))).to(dtype).cuda()
    pg.store(rows(sum(prompts), H), rows(sum(prompts), H), slots, *cache)
    src = [bounds[g] for g in (0, 1) for _ in range(answers[g])]
    dst = [bounds[g] + 1 + k for g in (0, 1) for k in range(answers[g])]
    pg.fork(i(src), i(dst), kv, table, free, nf, nf, *cache)
    assert kv.tolist() == [prompts[0]] * bounds[1] + [prompts[1]] * (B - bounds[1])
    groups, shared = i(bounds), i([n // page * page for n in prompts])
    lam, gain = torch.from_numpy(rng.uniform(0.2, 0.8, HQ)).float().cuda(), torch.from_numpy(rng.uniform(0.5, 1.5, 128)).float().cuda()
    # one step, captured: a token of every row that is still there
    step_new, slots = i([1] * B), i([0] * B)
    k_new, v_new, q = rows(B, H), rows(B, H), rows(B, HQ)
    out, out_diff = torch.zeros_like(q), torch.zeros_like(q)
    ws = [torch.zeros(n, dtype=torch.uint8, device="cuda") for n in (pg.attn_shared_bytes(B, 2), pg.attn_diff_bytes(B, B))]

    def step():
        pg.tables(kv, step_new, table, free, nf, q_start, kv, slots, nf)
        pg.store(k_new, v_new, slots, *cache)
        pg.attn_shared(q, kv, table, groups, shared, *cache, out, ws=ws[0])
        pg.attn_diff(q, kv, table, *cache, lam, out_diff, gain=gain, eps=1e-5, ws=ws[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()

    def check(what):
        torch.cuda.synchronize()
        lens = kv.tolist()
        K, V = pg.load(kv, table, *cache, max(lens))
        for b in range(B):
            for h in range(H):
                hs, n = slice(h * G, (h + 1) * G), lens[b]
                if n == 0:
                    assert not out[b].any() and not out_diff[b].any()
                    continue
                k, v = K[b, h, :n].double(), V[b, h, :n].double()          # (codes times powers of two: exact in either type)
                want, tol = attention("f32" if dtype == torch.float32 else "wide", q[b, hs], k, v, torch.full((G,), n, device="cuda"), 1 / math.sqrt(128))
                close(out[b, hs], want, tol, (what, b, h))
                expect(out_diff[b:b + 1, hs], "f32" if dtype == torch.float32 else "bf16", q[b:b + 1, hs], k, v, torch.full((1,), n, device="cuda"), 0.125, lam[hs],
                       gain, 1e-5, (what, b, h))
        named = {p for t, row in zip(lens, table[:, :14].tolist()) for p in row[:ref.pages_of(t, page)]}
        left = free.tolist()[:nf.item()]
        assert len(set(left)) == len(left) and named | set(left) == set(range(n_pages)) and not named & set(left), what
    check("first step")
    for n in range(3):
        for x in (k_new, v_new, q):
            x.copy_(rows(*x.shape[:2]))
        graph.replay()
        check(("answers", n))
    ended = np.zeros(B, int)
    ended[[bounds[0] + 1, bounds[1]]] = -1                   # an answer, and the row that the second prompt came in
    pg.release(kv, i(ended), table, free, nf, kv, nf)
    step_new.copy_(i(np.where(ended < 0, 0, 1)))
    pg.compact(kv, table, table, free, nf, new_id, *cache)
    assert nf.item() == n_pages - len({p for t, row in zip(kv.tolist(), table[:, :14].tolist()) for p in row[:ref.pages_of(t, page)]})
    # the rows that go on have a token each, those that ended none: a token's place is no longer its row
    alive = [b for b in range(B) if ended[b] == 0]
    k_few, v_few, few = rows(len(alive), H), rows(len(alive), H), i([0] * len(alive))
    pg.tables(kv, step_new, table, free, nf, q_start, kv, few, nf)
    pg.store(k_few, v_few, few, *cache)
    pg.attn_shared(q, kv, table, groups, shared, *cache, out)
    pg.attn_diff(q, kv, table, *cache, lam, out_diff, gain=gain, eps=1e-5)
    check("after the pool was compacted")
    assert kv.tolist()[1] == 0 and kv.tolist()[bounds[1]] == 0 and pg.device_status() == 0
