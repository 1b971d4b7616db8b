"""Bounded waits of fef_hidden_transform running out (needs a B200).

As in test_gpu_wait_timeout_products.py, with the test build of the library (-DFEF_TEST_HOOKS): the first CTA's producer stops
before a stage, so nothing is copied and nothing arrives for it, and the waits for that stage end after the limit that the test
sets.  Every role of every CTA that waits for it has to give up, what was issued has to finish before the tensor memory goes back,
the call reports FEF_ERR_TIMEOUT, and the next call is exact.  Nothing faults, traps or hangs."""
import ctypes
import time

import pytest
import torch

pytestmark = pytest.mark.gpu

FEF_ERR_TIMEOUT = 6
vp, i32, i64, u64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_uint64


@pytest.fixture(scope="module")
def hooks():
    from paper_2605_14305_b200 import _build

    L = ctypes.CDLL(_build.build_test_hooks())
    L.fef_hidden_transform.argtypes = [vp, i64, vp, vp, vp, i64, i32, i32, i32, i32, vp, i64, i32, vp, vp]
    L.fef_hidden_transform.restype = i32
    L.fef_test_withhold_transform_once.argtypes, L.fef_test_withhold_transform_once.restype = [i32, u64], None
    return L


# a cluster that shares a tile's depth, a CTA with several tiles, pairs of CTAs (the first stages, later ones, after the ring has turned)
@pytest.mark.parametrize("rows,n,d,stage", [(1, 4096, 4096, 0), (40, 2048, 4096, 3), (40, 2048, 4096, 9), (300, 40000, 256, 0), (300, 40000, 256, 13),
                                            (2048, 4096, 1024, 0), (2048, 4096, 1024, 5), (2048, 4096, 1024, 25)])
def test_withheld_stage(hooks, rows, n, d, stage):
    import paper_2605_14305_b200 as fef

    fef.load(build_if_missing=True)
    g = torch.Generator(device="cuda").manual_seed(rows + stage)
    h = torch.randn((rows, d), generator=g, device="cuda").to(torch.bfloat16)
    w = (torch.randn((n, d), generator=g, device="cuda") * d ** -0.5).to(torch.bfloat16)
    want, _ = fef.fef_hidden_transform(h, w, activation="silu")
    out = torch.zeros_like(want)
    status = torch.full((1,), 77, dtype=torch.int32, device="cuda")

    def call():
        return hooks.fef_hidden_transform(h.data_ptr(), d, w.data_ptr(), None, None, 0, rows, n, d, 2, out.data_ptr(), n, 1,
                                          status.data_ptr(), torch.cuda.current_stream().cuda_stream)

    hooks.fef_test_withhold_transform_once(stage, 20_000_000)
    start = time.monotonic()
    assert call() == 0
    torch.cuda.synchronize()                         # the kernel returned
    assert time.monotonic() - start < 15.0
    assert int(status.item()) == FEF_ERR_TIMEOUT
    assert call() == 0
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and torch.equal(out, want)
