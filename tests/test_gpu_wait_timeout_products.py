"""A bounded wait of the tensor-core products running out (needs a B200).

As in test_gpu_wait_timeout.py, with the test build of the library (-DFEF_TEST_HOOKS): the first CTA's producer stops
before a stage, so nothing is copied and nothing arrives for it, and the waits for that stage end after their limit of one second.
Every role has to give up, what was issued has to finish before the tensor memory goes back, the call reports FEF_ERR_TIMEOUT,
and the next call is exact.  Nothing faults, traps or hangs."""
import ctypes
import time

import pytest
import torch

pytestmark = pytest.mark.gpu

FEF_ERR_TIMEOUT = 6
vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t


@pytest.fixture(scope="module")
def hooks():
    from paper_2605_14305_b200 import _build

    L = ctypes.CDLL(_build.build_test_hooks())
    L.fef_lmhead_logits_quantized.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, vp, i64, i32, vp, sz, vp, vp]
    L.fef_lmhead_logits_quantized.restype = i32
    L.fef_lmhead_logits.argtypes = [vp, vp, i32, i32, i32, vp, i64, vp, vp]
    L.fef_lmhead_logits.restype = i32
    for f in (L.fef_test_withhold_product_block_once, L.fef_test_withhold_gemm_stage_once):
        f.argtypes, f.restype = [i32], None
    return L


@pytest.mark.parametrize("rows", [40, 200])          # (two pipelines of 64 rows, one of 128)
@pytest.mark.parametrize("block", [0, 3, 20])
def test_product_of_the_4_bit_layer(hooks, rows, block):
    import paper_2605_14305_b200 as fef

    V, d, group = 120000, 1024, 64                   # (eight blocks a tile, several tiles a CTA: number 20 comes after the ring has turned)
    fef.load(build_if_missing=True)
    g = torch.Generator(device="cuda").manual_seed(rows)
    layer = fef.fef_lmhead_quantize((torch.randn((V, d), generator=g, device="cuda") * 0.1).to(torch.bfloat16), group, True)
    hidden = torch.randn((rows, d), generator=g, device="cuda").to(torch.bfloat16)
    want, _ = fef.fef_lmhead_logits_quantized(hidden, layer)
    torch.cuda.synchronize()
    out = torch.zeros_like(want)
    need = fef.fef_lmhead_logits_quantized_workspace_bytes(rows, V, d, group)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call():
        return hooks.fef_lmhead_logits_quantized(hidden.data_ptr(), layer.packed.data_ptr(), layer.scale.data_ptr(),
                                                 layer.zero.data_ptr(), rows, V, d, group, out.data_ptr(), out.shape[1], 0,
                                                 ws.data_ptr(), ws.numel(), status.data_ptr(), torch.cuda.current_stream().cuda_stream)

    hooks.fef_test_withhold_product_block_once(block)
    start = time.monotonic()
    assert call() == 0
    torch.cuda.synchronize()                         # the kernels returned
    assert time.monotonic() - start < 10.0
    assert int(status.item()) == FEF_ERR_TIMEOUT
    assert call() == 0                               # the same stream, scratch and output
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and torch.equal(out[:, :V], want[:, :V])


@pytest.mark.parametrize("stage", [0, 2, 30])      # (of the 40 that the first CTA takes, through a ring of a few)
def test_product_of_the_16_bit_layer(hooks, stage):
    import paper_2605_14305_b200 as fef

    rows, V, d = 300, 60000, 512
    fef.load(build_if_missing=True)
    g = torch.Generator(device="cuda").manual_seed(stage)
    weight = (torch.randn((V, d), generator=g, device="cuda") * 0.1).to(torch.bfloat16)
    hidden = torch.randn((rows, d), generator=g, device="cuda").to(torch.bfloat16)
    want = torch.zeros((rows, V), device="cuda")
    fef.fef_lmhead_logits(hidden, weight, out=want)
    out = torch.zeros_like(want)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call():
        return hooks.fef_lmhead_logits(hidden.data_ptr(), weight.data_ptr(), rows, V, d, out.data_ptr(), V, status.data_ptr(),
                                       torch.cuda.current_stream().cuda_stream)

    hooks.fef_test_withhold_gemm_stage_once(stage)
    start = time.monotonic()
    assert call() == 0
    torch.cuda.synchronize()
    assert time.monotonic() - start < 10.0
    assert int(status.item()) == FEF_ERR_TIMEOUT
    assert call() == 0
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and torch.equal(out, want)
