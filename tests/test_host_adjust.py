"""Argument checks of fef_logits_adjust that need no GPU."""
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
    lib = fef.load()
    A, FAR = 0x1000, 0x10000000

    def adjust(logits=A, out=FAR, B=2, K=4, V=64, ld=64, dt=0, tokens=A, L=8, prompt=None, drafts=None, row_len=None, pen=A,
               bias=None, bias_stride=0, allowed=None, sb=0, sk=0, T=1.0, norm=None, ws=None, wsb=0):
        return lib.fef_logits_adjust(logits, out, B, K, V, ld, dt, tokens, L, prompt, drafts, row_len, pen, bias, bias_stride,
                                     allowed, sb, sk, T, norm, ws, wsb, None)

    bad = fef.FEF_ERR_INVALID_ARG
    assert adjust(dt=2) == fef.FEF_ERR_DTYPE
    assert adjust(logits=None) == bad and adjust(out=None) == bad
    assert adjust(B=0) == bad and adjust(B=65536) == bad and adjust(K=0) == bad and adjust(K=65) == bad
    assert adjust(V=0) == bad and adjust(ld=60) == bad and adjust(V=(1 << 28) + 1, ld=1 << 29) == bad
    assert adjust(L=-1) == bad and adjust(L=(1 << 24) + 1) == bad and adjust(tokens=None) == bad
    for T in (-1.0, float("nan"), float("inf")):
        assert adjust(T=T) == bad
    assert adjust(bias=A, bias_stride=63) == bad and adjust(bias=A, bias_stride=-64) == bad
    assert adjust(allowed=A, sb=1) == bad and adjust(allowed=A, sk=1) == bad and adjust(allowed=A, sk=-2) == bad
    assert adjust(out=A + 64) == bad                                # overlaps, but is not in place
    assert adjust(out=A + 2 * 4 * 64 * 4 - 16) == bad
    assert adjust(logits=A + 4) == fef.FEF_ERR_ALIGNMENT and adjust(out=FAR + 8) == fef.FEF_ERR_ALIGNMENT
    assert adjust(V=10, ld=10) == fef.FEF_ERR_ALIGNMENT
    assert adjust(tokens=A + 2) == fef.FEF_ERR_ALIGNMENT and adjust(norm=A + 4, ws=A, wsb=1 << 20) == fef.FEF_ERR_ALIGNMENT
    need = fef.fef_logits_adjust_workspace_bytes(2, 4, 64)
    assert need >= 2 * 4 * 8 and fef.fef_logits_adjust_workspace_bytes(0, 4, 64) == 0
    assert adjust(norm=A) == fef.FEF_ERR_WORKSPACE
    assert adjust(norm=A, ws=A, wsb=need - 1) == fef.FEF_ERR_WORKSPACE
    assert adjust(norm=A, ws=A + 16, wsb=1 << 20) == fef.FEF_ERR_WORKSPACE
    # valid calls get as far as the missing device
    assert adjust() == fef.FEF_ERR_CUDA and adjust(out=A) == fef.FEF_ERR_CUDA
    assert adjust(out=A + 2 * 4 * 64 * 4) == fef.FEF_ERR_CUDA
    assert adjust(tokens=None, L=0) == fef.FEF_ERR_CUDA and adjust(norm=A, ws=A, wsb=need) == fef.FEF_ERR_CUDA
    with pytest.raises(RuntimeError):
        fef.fef_logits_adjust(torch.zeros(1, 1, 8))
