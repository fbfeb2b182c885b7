"""Shared pages and differential attention at the edges of what their calls accept: starts that are any int32, steps without
forks, every wrong table entry."""
import numpy as np
import pytest
import torch

import pages_ref as ref
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
