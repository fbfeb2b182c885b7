"""A step in which requests are refused, as a server runs it: tables, store, attention."""
import numpy as np
import pytest
import torch

import pages_ref as ref
from test_gpu_pages_precision import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fk():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2507_20030_b200 import binding, build
    build.build()
    binding.load()
    return binding


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("t,n,free,room", [
    ([30, 40, 31, 20], [1, 30, 1, 1], 1, 33),          # the second needs two pages of one; the others stay inside theirs or wait
    ([30, 40, 31, 20], [9, 30, 40, 1], 9, 80),         # the third passes its table row
    ([30, 40, 31, 20], [9, 30, 5, 30], 9, 41),         # the third and the fourth pass n_tokens
])
def test_requests_beside_refused_ones(fk, dtype, t, n, free, room):
    rng = np.random.default_rng(free)
    page, W, H, G, B = 16, 4, 2, 4, 4
    n_pages = 20
    perm = rng.permutation(n_pages)
    table = np.full((B, W), -1)
    at = 0
    for b in range(B):
        k = ref.pages_of(t[b], page)
        table[b, :k] = perm[at:at + k]
        at += k
    stack = np.full(n_pages, -1)
    stack[:free] = perm[at:at + free]
    want = ref.tables(t, n, table.tolist(), stack.tolist(), free, room, page)
    w_table, _, _, w_start, w_kv, w_slots = want
    refused = [b for b in range(B) if w_kv[b] == t[b]]
    assert refused and len(refused) < B
    codes = [np.zeros((n_pages, H, page, 128), dtype=np.uint8) for _ in range(2)]
    scales = [np.full((n_pages, H), 2.0 ** -6) for _ in range(2)]
    for c in codes:
        c[:] = ref.encode(rng.standard_normal(c.shape) * 100.0)
    new = [torch.from_numpy(rng.standard_normal((room, H, 128))).to(dtype) for _ in range(2)]
    q = torch.from_numpy(rng.standard_normal((room, H * G, 128))).to(dtype).cuda()
    pg = fk.Pages(n_kv_heads=H, n_q_heads=H * G, page_size=page, n_pages=n_pages, max_pages=W, max_batch=B,
                  kv_dtype=fk.BF16 if dtype == torch.bfloat16 else fk.F32)
    d_c, d_s = [ref.cuda8(c) for c in codes], [ref.cuda32(s) for s in scales]
    kv, d_table, d_free, nf = ref.ints(t), ref.ints(table), ref.ints(stack), ref.ints([free])
    start, slots = ref.ints([0] * (B + 1)), ref.ints([0] * room)
    pg.tables(kv, ref.ints(n), d_table, d_free, nf, start, kv, slots, nf)
    pg.store(new[0].cuda(), new[1].cuda(), slots, *d_c, *d_s)
    out = torch.full_like(q, 7.0)
    pg.attn(q, kv, d_table, *d_c, *d_s, out, q_start=start)
    assert kv.tolist() == w_kv and slots.tolist() == w_slots and start.tolist() == w_start
    past = [b for b in range(B) if w_start[b + 1] > room]
    assert pg.device_status() == (0x105 if past else 0)
    for k in range(2):
        codes[k], scales[k] = ref.store(new[k].double().numpy(), w_slots, codes[k], scales[k], page)
        assert np.array_equal(d_c[k].view(torch.uint8).cpu().numpy(), codes[k])
    kind = "f32" if dtype == torch.float32 else "wide" if room * G > 8 * B else "bf16"
    for b in range(B):
        rows = slice(w_start[b], w_start[b + 1])
        if b in past:
            assert bool((out[rows] == 7.0).all())              # left as they were
            continue
        if n[b] < 1 or b in refused and n[b] > w_kv[b]:
            continue
        K, V = [torch.from_numpy(ref.rows_of(codes[k], scales[k], w_table[b], w_kv[b], page)).cuda() for k in range(2)]
        seen = w_kv[b] - n[b] + 1 + torch.arange(n[b], device="cuda").repeat_interleave(G)     # refused ones: of their older tokens
        for h in range(H):
            hs = slice(h * G, (h + 1) * G)
            check(kind, out[rows, hs].reshape(-1, 128), q[rows, hs].reshape(-1, 128), K[h], V[h], seen)
