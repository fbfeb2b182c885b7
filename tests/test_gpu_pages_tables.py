"""Block tables of steps without tokens: requests that only wait or finish."""
import numpy as np
import pytest
import torch

import pages_ref as ref
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


@pytest.mark.parametrize("B", [1, 300, 1024, 1025, 1500])
@pytest.mark.parametrize("finish", ["all", "some", "none"])
def test_steps_without_tokens(fk, B, finish):
    rng = np.random.default_rng(B)
    page, W = 16, 4
    t = rng.integers(0, W * page + 1, B)
    n = {"all": np.full(B, -1), "none": np.zeros(B, dtype=np.int64), "some": -rng.integers(0, 2, B)}[finish]
    held = [ref.pages_of(int(x), page) for x in t]
    n_pages = max(1, sum(held))
    perm = rng.permutation(n_pages)
    table = np.full((B, W), -7)
    at = 0
    for b, k in enumerate(held):
        table[b, :k] = perm[at:at + k]
        at += k
    free = np.full(n_pages, -9)
    want = ref.tables(t.tolist(), n.tolist(), table.tolist(), free.tolist(), 0, 0, page)
    pg = fk.Pages(n_kv_heads=1, n_q_heads=1, page_size=page, n_pages=n_pages, max_pages=W, max_batch=B)
    d_t, d_n, d_table, d_free, d_nf = ref.ints(t), ref.ints(n), ref.ints(table), ref.ints(free), ref.ints([0])
    q_start, slots = Guarded((B + 1,), torch.int32, -5), torch.zeros(0, dtype=torch.int32, device="cuda")
    pg.tables(d_t, d_n, d_table, d_free, d_nf, q_start.t, d_t, slots, d_nf)
    for name, a, b in zip(("table", "free", "n_free", "q_start", "kv_len"), (d_table, d_free, d_nf, q_start.t, d_t), want):
        assert np.array_equal(a.cpu().numpy(), np.asarray(b).reshape(a.shape)), name
    q_start.check("q_start")
    assert pg.device_status() == 0
