"""Argument checks of fef_hidden_transform that need no GPU."""
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
    H, W, R, O = 0x100000, 0x200000, 0x300000, 0x400000
    bad, align, most = fef.FEF_ERR_INVALID_ARG, fef.FEF_ERR_ALIGNMENT, fef.FEF_MAX_TRANSFORM

    def f(hidden=H, ldh=64, weight=W, bias=None, res=None, ldr=0, rows=4, n=32, d=64, act=0, out=O, ldo=32, dt=1, status=None):
        return lib.fef_hidden_transform(hidden, ldh, weight, bias, res, ldr, rows, n, d, act, out, ldo, dt, status, None)

    assert f(dt=2) == fef.FEF_ERR_DTYPE
    assert f(hidden=None) == bad and f(weight=None) == bad and f(out=None) == bad
    assert f(rows=0) == bad and f(n=0) == bad and f(d=0) == bad and f(d=60) == bad and f(d=-8) == bad
    assert f(rows=most + 1) == bad and f(n=most + 1, ldo=1 << 21) == bad and f(d=most + 8, ldh=1 << 21) == bad
    assert f(ldh=56) == bad and f(ldo=31) == bad and f(res=R, ldr=31) == bad and f(act=-1) == bad and f(act=5) == bad
    assert f(ldo=1 << 62) == bad and f(ldh=1 << 62) == bad and f(res=R, ldr=1 << 62) == bad
    assert f(hidden=H + 8) == align and f(weight=W + 8) == align and f(ldh=68) == align and f(bias=W + 1) == align
    assert f(res=R + 1, ldr=32) == align and f(out=O + 1) == align and f(out=O + 2, dt=0) == align and f(status=O + 2) == align
    # the output over the hidden states, the weights, the bias, another part of the residual
    assert f(out=H + 64 * 2 * 3) == bad and f(out=W - 64) == bad and f(bias=O + 62) == bad
    assert f(res=O + 64, ldr=32) == bad and f(res=O, ldr=40) == bad and f(res=O, ldr=32, dt=0) == bad
    # the output that is the residual; the ends of the ranges; a residual just behind the output
    for ok in (f(), f(res=O, ldr=32), f(res=O, ldr=99, rows=1), f(res=O + 4 * 32 * 2, ldr=32), f(out=O + 2), f(ldh=72, ldo=33),
               f(rows=1, n=1, d=8, ldh=8, ldo=1, act=4, dt=0), f(bias=R, res=R + 64, ldr=32, status=R)):
        assert ok == fef.FEF_ERR_CUDA
    # columns of one buffer: side by side, or over one another by two bytes; the hidden states on either side of the output
    wide = dict(ldh=96, ldo=96, ldr=96)
    for ok in (f(out=H + 128, **wide), f(out=H - 64, **wide), f(out=H - 192 - 64, **wide), f(out=O, res=O + 64, **wide),
               f(out=O, res=O + 128, **wide), f(out=O + 128, res=O, **wide)):
        assert ok == fef.FEF_ERR_CUDA
    for out in (H + 126, H - 62, H + 192 - 62, H + 192 * 3 + 126):
        assert f(out=out, **wide) == bad
    for res in (O + 62, O + 130, O - 62, O + 192 - 62, O + 192):
        assert f(out=O, res=res, **wide) == bad
    with pytest.raises(RuntimeError):
        fef.fef_hidden_transform(torch.zeros(1, 8), torch.zeros(1, 8))
