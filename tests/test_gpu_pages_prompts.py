"""Whole prompts through the paged cache's attention, and steps with many new tokens captured into graphs."""
import numpy as np
import pytest
import torch

import pages_ref as ref
from test_gpu_pages_precision import check, queries, sequence

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fk():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2507_20030_b200 import binding, build
    build.build()
    binding.load()
    return binding


@pytest.mark.parametrize("dtype,n,before,page", [
    (torch.bfloat16, 17500, 0, 64),         # more blocks of 128 columns than are shared out evenly
    (torch.bfloat16, 17000, 900, 16),
    (torch.float32, 1300, 77, 32),          # the same with eight columns a block
    (torch.bfloat16, 9000, 0, 128),         # fewer: shared out
])
def test_a_whole_prompt(fk, dtype, n, before, page):
    """One sequence's tokens all at once, over `before` cached ones: rows from both ends and the middle."""
    rng = np.random.default_rng(n)
    G, total = 8, before + n
    table, codes, scales, (K, V) = sequence(rng, total, 1, page, 9.0, "zero")
    q = queries(rng, n, G, 9.0, dtype)
    pg = fk.Pages(n_kv_heads=1, n_q_heads=G, page_size=page, n_pages=len(table), max_pages=len(table), max_batch=2,
                  kv_dtype=fk.BF16 if dtype == torch.bfloat16 else fk.F32)
    out = torch.full((n + 5, G, 128), 7.0, dtype=dtype, device="cuda")
    q = torch.cat([q, q[:5]])
    # beside it a sequence without new tokens; padding behind
    pg.attn(q, ref.ints([total, 0]), ref.ints(np.tile(table, (2, 1))), *codes, *scales, out, q_start=ref.ints([0, n, n]))
    assert pg.device_status() == 0
    assert bool((out[n:] == 7.0).all())
    kind = "wide" if dtype == torch.bfloat16 else "f32"
    for i0 in (0, 1, 127, n // 2, n - 300, n - 30):
        rows = slice(i0, i0 + 30)
        seen = (before + torch.arange(i0, i0 + 30, device="cuda") + 1).repeat_interleave(G)
        check(kind, out[rows].reshape(-1, 128), q[rows].reshape(-1, 128), K[0], V[0], seen)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_steps_with_many_new_tokens_replayed(fk, dtype):
    """Tables (two kernels), store and attention (with its join) of a step of many tokens, captured once and replayed on other
    lengths and tokens: equal to eager calls bit for bit."""
    rng = np.random.default_rng(6)
    H, G, page, W, B, n_pages, room = 2, 4, 16, 300, 3, 700, 2500
    steps = [[2200, 40, 200], [1, 1500, 3], [900, -1, 1500]]
    data = [[torch.from_numpy(rng.standard_normal((room, h, 128))).to(dtype).cuda() for h in (H, H, H * G)] for _ in steps]

    def serve(graph):
        pg = fk.Pages(n_kv_heads=H, n_q_heads=H * G, page_size=page, n_pages=n_pages, max_pages=W, max_batch=B,
                      kv_dtype=fk.BF16 if dtype == torch.bfloat16 else fk.F32)
        cache = pg.alloc()
        for c in cache[:2]:
            c.view(torch.uint8).zero_()
        for s in cache[2:]:
            s.fill_(1.0)
        t_len, table = ref.ints([0] * B), ref.ints(np.full((B, W), -1))
        free, n_free, start, slots = ref.ints(np.arange(n_pages)), ref.ints([n_pages]), ref.ints([0] * (B + 1)), ref.ints([0] * room)
        n_new = ref.ints([0] * B)
        k, v, q = [torch.zeros_like(x) for x in data[0]]
        out = torch.zeros_like(q)

        def step():
            pg.tables(t_len, n_new, table, free, n_free, start, t_len, slots, n_free)
            pg.store(k, v, slots, *cache)
            pg.attn(q, t_len, table, *cache, out, q_start=start)

        captured, got = None, []
        for new, d in zip(steps, data):
            n_new.copy_(ref.ints(new))
            for to, x in zip((k, v, q), d):
                to.copy_(x)
            out.fill_(7.0)
            if graph and captured is None:
                torch.cuda.synchronize()
                captured = torch.cuda.CUDAGraph()
                with torch.cuda.graph(captured):
                    step()
            if graph:
                captured.replay()
            else:
                step()
            torch.cuda.synchronize()
            got.append(out.clone())
        assert pg.device_status() == 0
        return got, [c.view(torch.uint8) for c in cache[:2]], list(cache[2:]), (t_len, n_free)

    a, b = serve(False), serve(True)
    assert a[3][0].tolist() == [3101, 0, 1703] and torch.equal(a[3][0], b[3][0]) and torch.equal(a[3][1], b[3][1])
    for x, y in zip(a[0] + a[1] + a[2], b[0] + b[1] + b[2]):
        assert torch.equal(x, y)
    assert bool((a[0][1][1504:] == 7.0).all()) and not bool((a[0][1][:1504] == 7.0).all(dim=2).any())
