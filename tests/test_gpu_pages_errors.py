"""An error that one call of the paged cache reports is not reported again by the next."""
import ctypes

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


def test_an_error_is_reported_once(fk):
    """The status word cannot be read while its stream is captured: that call fails, on the host, and the next one does not."""
    pg = fk.Pages(n_kv_heads=1, n_q_heads=1, page_size=16, n_pages=2, max_pages=2, max_batch=1)
    cache = pg.alloc()
    k = torch.ones((3, 1, 128), dtype=torch.bfloat16, device="cuda")
    slots = ref.ints([0, 1, 2])
    rt = ctypes.CDLL("libcudart.so.12")
    rt.cudaStreamBeginCapture.argtypes = [ctypes.c_void_p, ctypes.c_int]
    rt.cudaStreamEndCapture.argtypes = [ctypes.c_void_p, ctypes.POINTER(ctypes.c_void_p)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = ctypes.c_void_p()
    assert rt.cudaStreamBeginCapture(side.cuda_stream, 2) == 0          # relaxed: nothing else in the process is affected
    status = pg.device_status(stream=side)
    assert rt.cudaStreamEndCapture(side.cuda_stream, ctypes.byref(graph)) != 0 and not graph.value
    rt.cudaGetLastError()
    assert status == -6
    pg.store(k, k, slots, *cache)
    assert pg.device_status() == 0
    assert bool((cache[0][0, 0, :3].float() * cache[2][0, 0] == 1.0).all())
