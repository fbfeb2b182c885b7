"""Shared pages and differential attention without a GPU: refusals of the C entries and of the binding, the reference's own pins."""
import numpy as np
import pytest
import torch

import pages_share_ref as share


@pytest.fixture(scope="module")
def fk():
    from paper_2507_20030_b200 import binding, build
    build.build()
    binding.load()
    return binding


class Recorder:
    """Stands for the library: writes down each call and says yes."""
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_bytes"):
                return 64
            self.calls.append((name, args))
            return 0
        return call


def bare(fk, **kw):
    pg = object.__new__(fk.Pages)
    pg.__dict__.update(dict(n_kv_heads=2, n_q_heads=4, page_size=16, n_pages=3, max_pages=4, max_batch=2, kv_dtype=fk.BF16, head_dim=128,
                            device=torch.device("cpu"), _h=None, _lib=Recorder()), **kw)
    pg._shapes()
    pg._on = lambda stream: 77
    return pg


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def refused_one_by_one(call, good, names, bad_of):
    """call(**good) goes through; with one tensor in a wrong shape, type or layout a ValueError names it."""
    call(**good)
    for name in names:
        for bad in bad_of(good[name]):
            with pytest.raises(ValueError, match=name):
                call(**{**good, name: bad})


def wrong(t):
    return [t.double(), t[..., :-1], torch.zeros((2,) + tuple(t.shape), dtype=t.dtype)] + ([t.transpose(0, 1).contiguous().transpose(0, 1)] if t.dim() == 2 and min(t.shape) > 1 else [])


def test_null_handles_are_refused(fk):
    lib, z = fk.load(), None
    assert lib.faedkv_pages_fork(z, z, z, z, 0, 1, z, z, z, z, z, z, z, z, z, z, z) == -1
    assert lib.faedkv_pages_release(z, z, z, 1, z, z, z, z, z, z, z) == -1
    assert lib.faedkv_pages_compact(z, z, 1, z, z, z, z, z, z, z, z, z, z, z) == -1
    assert lib.faedkv_pages_attn_shared(z, z, 256, z, z, 1, 1, z, z, z, z, z, z, 0.0, z, z, 0, z) == -1
    assert lib.faedkv_pages_attn_diff(z, z, 256, z, 1, 1, z, z, z, z, z, z, 0.0, z, z, 0.0, z, z, 0, z) == -1
    assert lib.faedkv_pages_attn_shared_bytes(z, 1, 1) == 0 and lib.faedkv_pages_attn_diff_bytes(z, 1, 1) == 0
    assert lib.faedkv_pages_fork_bytes(z, 1, 1) == 0 and lib.faedkv_pages_release_bytes(z) == 0 and lib.faedkv_pages_compact_bytes(z) == 0


def test_binding_refuses_wrong_tensors_of_the_page_calls(fk):
    pg = bare(fk)
    codes, scale = torch.zeros(3, 2, 16, 128, dtype=torch.float8_e4m3fn), torch.zeros(3, 2)
    cache = dict(k_pages=codes, v_pages=codes, k_scale=scale, v_scale=scale)
    base = dict(kv_len=i32(2), table=i32(2, 4), free_pages=i32(3), n_free=i32(1))
    ws = torch.zeros(64, dtype=torch.uint8)
    ints = ["kv_len", "table", "free_pages", "n_free"]
    fork = dict(base, src=i32(2), dst=i32(2), length=i32(2), n_free_out=i32(1), ws=ws, **cache)
    refused_one_by_one(pg.fork, fork, [*ints[1:], "dst", "length", "n_free_out", *cache], wrong)
    release = dict(base, t_len=i32(2), n_new=i32(2), n_free_out=i32(1), ws=ws)
    refused_one_by_one(pg.release, release, [*ints, "n_new", "n_free_out"], wrong)
    compact = dict(base, table_out=i32(2, 4), new_id=i32(3), ws=ws, **cache)
    refused_one_by_one(pg.compact, compact, [*ints[1:], "table_out", "new_id", *cache], wrong)
    for call, args in ((pg.fork, fork), (pg.release, release), (pg.compact, compact)):      # (the recorder asks for 64 bytes)
        with pytest.raises(ValueError, match="ws"):
            call(**{**args, "ws": torch.zeros(8, dtype=torch.uint8)})
    assert {name for name, _ in pg._lib.calls} == {"faedkv_pages_fork", "faedkv_pages_release", "faedkv_pages_compact"}
    name, args = next(c for c in pg._lib.calls if c[0] == "faedkv_pages_fork")
    assert args == (None, fork["src"].data_ptr(), fork["dst"].data_ptr(), fork["length"].data_ptr(), 2, 2, fork["kv_len"].data_ptr(),
                    fork["table"].data_ptr(), fork["free_pages"].data_ptr(), fork["n_free"].data_ptr(), fork["n_free_out"].data_ptr(),
                    codes.data_ptr(), codes.data_ptr(), scale.data_ptr(), scale.data_ptr(), ws.data_ptr(), 77)


def test_binding_refuses_wrong_tensors_of_the_attention_calls(fk):
    pg = bare(fk)
    codes, scale = torch.zeros(3, 2, 16, 128, dtype=torch.float8_e4m3fn), torch.zeros(3, 2)
    cache = dict(k_pages=codes, v_pages=codes.clone(), k_scale=scale, v_scale=scale.clone())
    ws = torch.zeros(64, dtype=torch.uint8)
    rows = torch.zeros(2, 4, 128, dtype=torch.bfloat16)
    base = dict(q=rows, kv_len=i32(2), table=i32(2, 4), out=rows.clone(), ws=ws, **cache)
    shared = dict(base, group_start=i32(2), shared_len=i32(1))
    refused_one_by_one(pg.attn_shared, shared, ["q", "table", "group_start", "out", *cache], wrong)
    diff = dict(base, lam=torch.zeros(4), gain=torch.ones(128), q_start=i32(3))
    refused_one_by_one(pg.attn_diff, diff, ["q", "table", "q_start", "lam", "gain", "out", *cache], wrong)
    with pytest.raises(ValueError, match="one token for each of 2 rows"):
        pg.attn_shared(**{**shared, "q": torch.zeros(3, 4, 128, dtype=torch.bfloat16), "out": torch.zeros(3, 4, 128, dtype=torch.bfloat16)})
    for call, args in ((pg.attn_shared, shared), (pg.attn_diff, diff)):
        with pytest.raises(ValueError, match="ws"):
            call(**{**args, "ws": torch.zeros(8, dtype=torch.uint8)})
    calls = {name: args for name, args in pg._lib.calls}
    c = [cache[k].data_ptr() for k in ("k_pages", "v_pages", "k_scale", "v_scale")]
    ptr = {k: t.data_ptr() for k, t in {**shared, **diff}.items()}
    assert calls["faedkv_pages_attn_shared"] == (None, ptr["q"], 512, ptr["group_start"], ptr["shared_len"], 1, 2, ptr["kv_len"], ptr["table"], *c, 0.0,
                                                 ptr["out"], ptr["ws"], 64, 77)
    assert calls["faedkv_pages_attn_diff"] == (None, ptr["q"], 512, ptr["q_start"], 2, 2, ptr["kv_len"], ptr["table"], *c, 0.0, ptr["lam"],
                                               ptr["gain"], 0.0, ptr["out"], ptr["ws"], 64, 77)


def test_reference_fork_release_compact_by_hand():
    kv, table = [37, 16, 0, 0, 0], [[4, 7, 9], [2, 0, 0]] + [[0] * 3] * 3
    kv2, table2, n, copies = share.fork([0, 1, 0], [2, 3, 4], [37, 99, 33], kv, table, [1, 3, 5, 0, 0, 0, 0, 0, 0, 0], 3, 16)
    assert kv2 == [37, 16, 37, 16, 33] and n == 1 and copies == [(9, 5, 5), (9, 3, 1)]
    assert table2[2] == [4, 7, 5] and table2[3][0] == 2 and table2[4] == [4, 7, 3]
    free, n, kv3 = share.release(kv2, [0, -1, -1, 0, -1], table2, [1] + [0] * 9, 1, 16)
    assert free[:n] == [1, 5, 3] and kv3 == [37, 0, 0, 16, 0]              # 4 and 7 are request 0's still, 2 request 3's
    table4, free, n, new, moves = share.compact(kv3, table2, [0] * 10, 10, 16)
    assert moves == [(4, 0), (7, 1), (9, 3)] and table4[0] == [0, 1, 3] and table4[3][0] == 2 and n == 6 and free[:6] == [9, 8, 7, 6, 5, 4]
    assert new == [-1, -1, 2, -1, 0, -1, -1, 1, -1, 3]
