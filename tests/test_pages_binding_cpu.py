"""binding.Pages against a library that only records what it is called with."""
import pytest
import torch


@pytest.fixture(scope="module")
def fk():
    from paper_2507_20030_b200 import binding, build
    build.build()
    binding.load()
    return binding


class Recorder:
    def __init__(self):
        self.calls = []

    def faedkv_pages_load(self, *args):
        self.calls.append(args)
        return 0


def _bare(fk):
    pg = object.__new__(fk.Pages)
    pg.__dict__.update(n_kv_heads=2, n_q_heads=4, page_size=16, n_pages=3, max_pages=4, max_batch=2, kv_dtype=fk.BF16, head_dim=128,
                       device=torch.device("cpu"), _h=None, _lib=Recorder())
    pg._shapes()
    pg._on = lambda stream: 77
    return pg


def test_load_of_keys_or_values_alone(fk):
    """The C call takes either; the binding passes NULL for what is left out and refuses halves of one."""
    pg = _bare(fk)
    codes, scale = torch.zeros(3, 2, 16, 128, dtype=torch.float8_e4m3fn), torch.zeros(3, 2)
    kv, table = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 4, dtype=torch.int32)
    K, V = pg.load(kv, table, codes, None, scale, None, 5)
    assert V is None and K.shape == (2, 2, 5, 128)
    assert pg._lib.calls[-1] == (None, kv.data_ptr(), table.data_ptr(), 2, 5, codes.data_ptr(), None, scale.data_ptr(), None, K.data_ptr(), None, 77)
    K, V = pg.load(kv, table, None, codes, None, scale, 5)
    assert K is None
    assert pg._lib.calls[-1] == (None, kv.data_ptr(), table.data_ptr(), 2, 5, None, codes.data_ptr(), None, scale.data_ptr(), None, V.data_ptr(), 77)
    given = torch.zeros(2, 2, 5, 128, dtype=torch.bfloat16)
    K, V = pg.load(kv, table, codes, codes, scale, scale, 5, K_out=given)
    assert K is given and V.shape == given.shape
    n = len(pg._lib.calls)
    for args, kw in [((codes, None, None, None), {}), ((None, codes, scale, scale), {}), ((None, None, None, None), {}),
                     ((codes, None, scale, None), {"V_out": given}), ((codes, codes, scale, scale), {"K_out": given[:, :, :4]})]:
        with pytest.raises(ValueError):
            pg.load(kv, table, args[0], args[1], args[2], args[3], 5, **kw)
    assert len(pg._lib.calls) == n
