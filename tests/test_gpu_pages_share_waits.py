"""The bounded waits of attention over shared pages and of differential attention run out: the kernels leave a code and end."""
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


@pytest.mark.parametrize("form", ["shared rows", "shared", "shared f32", "diff decode", "diff rows", "diff one tile of rows"])
@pytest.mark.parametrize("tile", [1, 2, 5])
def test_waits_that_run_out(fk, form, tile):
    """Waits limited to 1 ms and one warp's signal kept back at a tile: the kernel ends by itself, leaves a code, and the next call, hooks
    off, gives what the one before gave."""
    rng = np.random.default_rng(1)
    H, G, page, n = 2, 4, 64, 90000                       # more than six tiles for each CTA, whatever the form
    B = 70 if form == "shared rows" else 2
    dtype = torch.float32 if "f32" in form else torch.bfloat16
    n_pages = ref.pages_of(n, page)
    pg = fk.Pages(n_kv_heads=H, n_q_heads=H * G, page_size=page, n_pages=n_pages, max_pages=4 * n_pages, max_batch=B,
                  kv_dtype=fk.BF16 if dtype == torch.bfloat16 else fk.F32)
    cache = [torch.randn((n_pages, H, page, 128), device="cuda").to(torch.float8_e4m3fn) for _ in range(2)]
    cache += [torch.full((n_pages, H), 0.5, device="cuda") for _ in range(2)]
    table = ref.ints(np.concatenate([np.tile(rng.permutation(n_pages), (B, 1)), np.full((B, 3 * n_pages), -1)], axis=1))
    kv = ref.ints([n] * B)
    new = {"diff rows": 40, "diff one tile of rows": 9}.get(form, 1)
    q = torch.randn((B * new, H * G, 128), device="cuda").to(dtype)
    out = torch.zeros_like(q)
    if "diff" in form:
        lam = torch.full((H * G,), 0.5, device="cuda")
        start = None if new == 1 else ref.ints([0, new, 2 * new])

        def call():
            pg.attn_diff(q, kv, table, *cache, lam, out, q_start=start)
    else:
        groups, share = ref.ints([0, B]), ref.ints([n // 64 * 64 - 6400])

        def call():
            pg.attn_shared(q, kv, table, groups, share, *cache, out)
    call()
    good = out.clone()
    assert pg.device_status() == 0
    pg.test_hooks(wait_limit_ns=1_000_000, withhold_tile=tile)
    t0 = time.perf_counter()
    call()
    torch.cuda.synchronize()
    assert time.perf_counter() - t0 < 2.0
    assert pg.device_status() in (0x41, 0x42, 0x43)
    pg.test_hooks()
    pg.reset_device_status()
    out.zero_()
    call()
    assert pg.device_status() == 0 and torch.equal(out, good)
