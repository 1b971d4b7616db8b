"""Argument checks of the 4-bit output layer's calls that need no GPU."""
import pytest
import torch

HAS_GPU = torch.cuda.is_available()


@pytest.fixture(scope="module")
def fef():
    import paper_2605_14305_b200 as lib

    lib.load(build_if_missing=True)
    return lib


@pytest.mark.skipif(HAS_GPU, reason="uses placeholder addresses; only meaningful where no kernel can launch")
def test_argument_checks_return_before_touching_the_device(fef):
    lib, A = fef.load(), 0x1000
    bad, align = fef.FEF_ERR_INVALID_ARG, fef.FEF_ERR_ALIGNMENT

    def quantize(w=A, V=10, d=128, g=32, p=A, s=A, z=A, st=None):
        return lib.fef_lmhead_quantize(w, V, d, g, p, s, z, st, None)

    def dequantize(p=A, s=A, z=A, V=10, d=128, g=32, out=A):
        return lib.fef_lmhead_dequantize(p, s, z, V, d, g, out, None)

    def product(h=A, p=A, s=A, z=A, rows=3, V=10, d=128, g=32, out=A, ldo=12, dt=0, ws=A, wsb=1 << 20, st=None):
        return lib.fef_lmhead_logits_quantized(h, p, s, z, rows, V, d, g, out, ldo, dt, ws, wsb, st, None)

    for call in (quantize, dequantize, product):
        assert call(p=None) == bad and call(s=None) == bad
        assert call(V=0) == bad and call(V=(1 << 28) + 1) == bad
        assert call(d=0) == bad and call(d=96, g=64) == bad and call(d=(1 << 20) + 128) == bad and call(d=-128) == bad
        for g in (0, 1, 16, 48, 256, -32):
            assert call(g=g) == bad
        assert call(p=A + 16) == align and call(s=A + 2) == align and call(z=A + 1) == align
        assert call() == fef.FEF_ERR_CUDA and call(z=None) == fef.FEF_ERR_CUDA
    assert quantize(w=None) == bad and quantize(w=A + 8) == align
    assert dequantize(out=None) == bad and dequantize(out=A + 4) == align
    assert product(h=None) == bad and product(out=None) == bad and product(rows=0) == bad and product(rows=(1 << 24) + 1) == bad
    assert product(ldo=8) == bad and product(ldo=11) == align and product(ldo=12, dt=1) == align and product(dt=2) == fef.FEF_ERR_DTYPE
    assert product(h=A + 2) == align and product(out=A + 8) == align
    for kw in (dict(ws=None), dict(ws=A + 16), dict(wsb=16000)):
        assert product(rows=40, **kw) == fef.FEF_ERR_WORKSPACE and product(rows=4, **kw) == fef.FEF_ERR_CUDA
    assert product(rows=40) == fef.FEF_ERR_CUDA
    need = fef.fef_lmhead_logits_quantized_workspace_bytes
    assert need(0, 10, 128, 32) == 0 and need(3, 10, 100, 32) == 0 and need(3, 10, 128, 48) == 0 and need(3, 10, 128, 32) == 256
    assert need(40, 10, 128, 32) >= 64 * 128 * 2
    with pytest.raises(RuntimeError):
        fef.fef_lmhead_quantize(torch.zeros((2, 32), dtype=torch.bfloat16))
