"""The bounded waits of the paged attention when they run out."""
import time

import numpy as np
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


@pytest.mark.parametrize("dtype,new", [(torch.bfloat16, None), (torch.float32, None), (torch.bfloat16, 40), (torch.float32, 3)])
@pytest.mark.parametrize("tile", [1, 2])
def test_waits_that_run_out(fk, dtype, new, tile):
    """Waits limited to 1 ms and one warp's signal kept back at a tile of every CTA: the kernel ends by itself, leaves a code, and the
    next call, hooks off, gives what the one before gave."""
    rng = np.random.default_rng(1)
    H, G, page, n, B = 2, 4, 64, 30000, 2
    n_pages = ref.pages_of(n, page)
    pg = fk.Pages(n_kv_heads=H, n_q_heads=H * G, page_size=page, n_pages=n_pages, max_pages=n_pages, max_batch=B,
                  kv_dtype=fk.BF16 if dtype == torch.bfloat16 else fk.F32)
    cache = [torch.randn((n_pages, H, page, 128), device="cuda").to(torch.float8_e4m3fn) for _ in range(2)]
    cache += [torch.full((n_pages, H), 0.5, device="cuda") for _ in range(2)]
    table = ref.ints([rng.permutation(n_pages) for _ in range(B)])
    q = torch.randn((B * (new or 1), H * G, 128), device="cuda").to(dtype)
    start = None if new is None else ref.ints([0, new, 2 * new])
    good, out = torch.zeros_like(q), torch.zeros_like(q)
    pg.attn(q, ref.ints([n] * B), table, *cache, good, q_start=start)
    assert pg.device_status() == 0
    pg.test_hooks(wait_limit_ns=1_000_000, withhold_tile=tile)
    t0 = time.perf_counter()
    pg.attn(q, ref.ints([n] * B), table, *cache, out, q_start=start)
    torch.cuda.synchronize()
    assert time.perf_counter() - t0 < 1.0
    assert pg.device_status() in (0x41, 0x42, 0x43)
    pg.test_hooks()
    pg.reset_device_status()
    pg.attn(q, ref.ints([n] * B), table, *cache, out, q_start=start)
    assert pg.device_status() == 0 and torch.equal(out, good)


def test_hooks_refuse_what_makes_no_sense(fk):
    pg = fk.Pages(1, 1, 16, 1, 1, 1)
    with pytest.raises(fk.FaedkvError):
        pg.test_hooks(0, -1)
    assert pg._lib.faedkv_pages_test_hooks(None, 0, 0) == -1
