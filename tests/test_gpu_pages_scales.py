"""Writes into pages whose scales the caller has set: not powers of two."""
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


@pytest.mark.parametrize("top", [448.0, 224.0])
def test_codes_under_a_scale_that_is_no_power_of_two(fk, top):
    """A token behind others in a page keeps the page's scale when the power of two that it needs is not larger (224: always; 448:
    seldom): its codes are those of the float32 quotient x / s, at the midpoints of neighbouring codes too, where a product
    with 1 / s would fall to either side."""
    rng = np.random.default_rng(0)
    n = 64
    mid = ((ref.VALUES[1:127] + ref.VALUES[:126]) / 2).astype(np.float32)
    mid = mid[mid < top]
    scales = rng.uniform(0.001, 3.0, n).astype(np.float32)
    scales[:4] = [3.3e38 / 512, 1.5e-37, 1.0 / 3.0, 0.1]
    x = np.zeros((n, 1, 128), dtype=np.float32)
    x[:, 0, :len(mid)] = scales[:, None] * mid[None, :]
    assert 0.3 < np.mean((x / scales[:, None, None])[:, 0, :len(mid)] == mid[None, :])     # ties are met
    need = np.array([ref.scale_for(float(np.abs(v).max())) for v in x], dtype=np.float32)
    want_s = np.maximum(scales, need)
    assert top == 448.0 or np.array_equal(want_s, scales)
    want = ref.encode((x / want_s[:, None, None]).astype(np.float64))
    pg = fk.Pages(n_kv_heads=1, n_q_heads=1, page_size=16, n_pages=n, max_pages=1, max_batch=1, kv_dtype=fk.F32)
    codes = [torch.zeros((n, 1, 16, 128), dtype=torch.uint8, device="cuda") for _ in range(2)]
    s = [torch.from_numpy(scales).cuda().view(n, 1).clone() for _ in range(2)]
    k = torch.from_numpy(x).cuda()
    pg.store(k, k, ref.ints(np.arange(n) * 16 + 3), *[c.view(torch.float8_e4m3fn) for c in codes], *s)
    for c, t in zip(codes, s):
        assert np.array_equal(t.cpu().numpy()[:, 0], want_s)
        assert np.array_equal(c[:, 0, 3].cpu().numpy(), want[:, 0])
    assert pg.device_status() == 0
