"""Memory that the paged cache's binding allocates belongs to the stream of the call."""
import pytest
import torch

import pages_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fk():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2507_20030_b200 import binding, build
    build.build()
    binding.load()
    return binding


@pytest.mark.parametrize("raw", [False, True])
def test_rows_and_workspaces_are_allocated_on_the_calls_stream(fk, raw, monkeypatch):
    pg = fk.Pages(n_kv_heads=2, n_q_heads=4, page_size=16, n_pages=4, max_pages=2, max_batch=1)
    cache = pg.alloc()
    k = torch.randn((20, 2, 128), device="cuda").to(torch.bfloat16)
    table, kv_len = ref.ints([[2, 1]]), ref.ints([20])
    pg.store(k, k, ref.ints([32 + i for i in range(16)] + [16 + i for i in range(4)]), *cache)
    q = torch.randn((1, 4, 128), device="cuda").to(torch.bfloat16)
    out = torch.empty_like(q)
    K, V = pg.load(kv_len, table, *cache, 24)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    handle = side.cuda_stream if raw else side
    seen, empty = [], torch.empty

    def recording(*args, **kw):
        seen.append(torch.cuda.current_stream().cuda_stream)
        return empty(*args, **kw)

    monkeypatch.setattr(torch, "empty", recording)
    K2, V2 = pg.load(kv_len, table, *cache, 24, stream=handle)
    pg.attn(q, kv_len, table, *cache, out, stream=handle)
    monkeypatch.undo()
    torch.cuda.synchronize()
    assert seen == [side.cuda_stream] * 3
    assert torch.equal(K, K2) and torch.equal(V, V2)
