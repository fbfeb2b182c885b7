"""Writes to the paged 8-bit cache with refused tokens (no slot, or one outside the pool) between those that are written."""
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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,H,n,pattern", [
    (16, 8, 1500, "10"),            # every second token refused
    (32, 8, 900, "1101"),
    (16, 4, 1200, "1000110101"),
    (128, 2, 4000, "12012"),        # 2: a slot behind the pool
])
def test_tokens_between_refused_ones(fk, dtype, page, H, n, pattern):
    """Several runs a CTA with an odd number of skipped tokens between them.  Magnitudes differ by 2^10 from one token to the next, so
    that a maximum taken from another run would show in the scale."""
    rng = np.random.default_rng(n + page)
    kind = [pattern[i % len(pattern)] for i in range(n)]
    n_pages = n + 1
    at = rng.permutation(n_pages)
    rows = rng.integers(0, page, n)
    slots = [{"1": int(at[i]) * page + int(rows[i]), "0": -1, "2": n_pages * page + i}[k] for i, k in enumerate(kind)]
    x = [rng.standard_normal((n, H, 128)) * 2.0 ** rng.integers(-10, 11, (n, H, 1)) for _ in range(2)]
    x = [torch.from_numpy(v).to(dtype) for v in x]
    pg = fk.Pages(n_kv_heads=H, n_q_heads=H, page_size=page, n_pages=n_pages, max_pages=1, max_batch=1,
                  kv_dtype=fk.BF16 if dtype == torch.bfloat16 else fk.F32)
    codes = [torch.zeros((n_pages, H, page, 128), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.full((n_pages, H), 2.0 ** -20, device="cuda") for _ in range(2)]
    for _ in range(5):
        for c, s in zip(codes, scales):
            c.zero_()
            s.fill_(2.0 ** -20)
        pg.store(x[0].cuda(), x[1].cuda(), ref.ints(slots), *[c.view(torch.float8_e4m3fn) for c in codes], *scales)
        for v, c, s in zip(x, codes, scales):
            v = v.double().numpy()
            want_s = np.full((n_pages, H), 2.0 ** -20)
            want_c = np.zeros((n_pages, H, page, 128), dtype=np.uint8)
            for i, k in enumerate(kind):
                if k == "1":
                    p, r = divmod(slots[i], page)
                    need = np.exp2(np.ceil(np.log2(np.abs(v[i]).max(axis=1) / 448.0)))
                    want_s[p] = need if r == 0 else np.maximum(need, want_s[p])
                    want_c[p, :, r] = ref.encode(v[i] / want_s[p][:, None])
            assert np.array_equal(s.cpu().numpy().astype(np.float64), want_s)
            assert np.array_equal(c.cpu().numpy(), want_c)
    assert pg.device_status() == (0x102 if "2" in pattern else 0)
