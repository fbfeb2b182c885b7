"""The paged 8-bit cache without a GPU: refusals of the C entries, the binding's shape checks, the reference's own pins."""
import ctypes

import numpy as np
import pytest
import torch

import pages_ref as ref


@pytest.fixture(scope="module")
def fk():
    from paper_2507_20030_b200 import binding, build
    build.build()
    binding.load()
    return binding


def test_create_refuses_bad_configs_before_touching_cuda(fk):
    lib = fk.load()
    good = dict(n_kv_heads=8, n_q_heads=32, head_dim=128, page_size=64, n_pages=100, max_pages=16, max_batch=4, kv_dtype=fk.BF16)
    h = ctypes.c_void_p()
    for key, bad, code in [("head_dim", 64, -4), ("page_size", 8, -4), ("page_size", 48, -4), ("page_size", 256, -4), ("n_pages", 0, -1),
                           ("max_pages", 0, -1), ("max_batch", 0, -1), ("max_batch", 65536, -3), ("kv_dtype", 2, -1), ("n_q_heads", 12, -4),
                           ("n_q_heads", 72, -4), ("n_kv_heads", 0, -1), ("n_pages", 1 << 25, -3), ("n_pages", 1 << 22, -3),
                           ("max_pages", (1 << 24) + 1, -3), ("n_q_heads", 0, -1)]:
        cfg = fk.PagesConfig(**{**good, key: bad})
        assert lib.faedkv_pages_create(ctypes.byref(cfg), ctypes.byref(h)) == code, (key, bad)
        assert not h.value
    cfg = fk.PagesConfig(**good)
    assert lib.faedkv_pages_create(None, ctypes.byref(h)) == -1
    assert lib.faedkv_pages_create(ctypes.byref(cfg), None) == -1


def test_null_handles_are_refused(fk):
    lib = fk.load()
    z = None
    assert lib.faedkv_pages_tables(z, z, z, 1, z, z, z, 1, z, z, z, z, z, z) == -1
    assert lib.faedkv_pages_store(z, z, z, 1024, z, 1, z, z, z, z, z) == -1
    assert lib.faedkv_pages_attn(z, z, 1024, z, 1, 1, z, z, z, z, z, z, 0.0, z, z, 0, z) == -1
    assert lib.faedkv_pages_load(z, z, z, 1, 1, z, z, z, z, z, z, z) == -1
    assert lib.faedkv_pages_device_status(z, z) == -1 and lib.faedkv_pages_reset_device_status(z, z) == -1
    assert lib.faedkv_pages_bytes(z) == 0 and lib.faedkv_pages_attn_bytes(z, 1, 1) == 0 and lib.faedkv_pages_launch_count(z) == 0
    lib.faedkv_pages_destroy(None)


def _bare(fk, **kw):
    pg = object.__new__(fk.Pages)
    pg.__dict__.update(dict(n_kv_heads=2, n_q_heads=4, page_size=16, n_pages=3, max_pages=4, max_batch=2, kv_dtype=fk.BF16, head_dim=128,
                            device=torch.device("cpu"), _h=None), **kw)
    pg._shapes()
    return pg


def test_binding_refuses_wrong_tensors_by_name(fk):
    pg = _bare(fk)
    x = torch.zeros(5, 2, 128, dtype=torch.bfloat16)
    assert pg._rows("k_new", x, 2)[1:] == (5, 256)
    wide = torch.zeros(5, 8, 128, dtype=torch.bfloat16)
    assert pg._rows("k_new", wide[:, 4:6], 2)[1:] == (5, 1024)          # a slice of a fused projection
    for bad in (x.float(), x[:, :1], x[..., :64], x.transpose(0, 1), torch.zeros(5, 256, dtype=torch.bfloat16), x[:1].expand(5, 2, 128),
                torch.zeros(5, 4, 128, dtype=torch.bfloat16)[:, ::2], torch.zeros(5, 2, 256, dtype=torch.bfloat16)[..., ::2]):
        with pytest.raises(ValueError, match="k_new"):
            pg._rows("k_new", bad, 2)
    codes, scale = torch.zeros(3, 2, 16, 128, dtype=torch.float8_e4m3fn), torch.zeros(3, 2)
    pg._cache(codes, codes, scale, scale)
    with pytest.raises(ValueError, match="v_pages"):
        pg._cache(codes, codes[:2], scale, scale)
    with pytest.raises(ValueError, match="k_pages"):
        pg._cache(codes.view(torch.uint8), codes, scale, scale)
    with pytest.raises(ValueError, match="v_scale"):
        pg._cache(codes, codes, scale, scale.double())
    with pytest.raises(ValueError, match="k_scale"):
        pg._cache(codes, codes, torch.zeros(2, 3).t(), scale)


def test_reference_rounding_agrees_with_the_definition():
    """The reference's own encoder against torch's cast on every midpoint and neighbour of the format."""
    v = ref.VALUES[:127]
    mid = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20), [449.0, 1e30]])
    x = np.concatenate([x, -x])
    want = torch.from_numpy(x).clamp(-448, 448).to(torch.float32).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(ref.VALUES[ref.encode(x)], want.astype(np.float64))
    assert ref.scale_for(448.0) == 1.0 and ref.scale_for(448.0001) == 2.0 and ref.scale_for(0.0) == 2.0 ** -126


def test_reference_attention_is_a_weighted_mean():
    rng = np.random.default_rng(1)
    table = ref.spread([5], 16, 2, 1, rng)
    kc, ks = ref.random_cache(rng, 2, 1, 16, [5], table)
    vc, vs = ref.random_cache(rng, 2, 1, 16, [5], table)
    out = ref.attn(np.zeros((1, 1, 128)), [0, 1], [5], table, kc, ks, vc, vs, 16)
    assert np.allclose(out[0, 0], ref.rows_of(vc, vs, table[0], 5, 16)[0].mean(axis=0), atol=1e-12)
