"""Argument checks of the calls on cut laws that need no GPU."""
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
    A = 0x1000
    bad, align = fef.FEF_ERR_INVALID_ARG, fef.FEF_ERR_ALIGNMENT

    def law(logits=A, row_len=None, B=2, K=4, V=64, ld=64, dt=0, T=1.0, k=A, p=A, m=A, norm=A, cut=A, cut_id=A, kept=A, status=A):
        return lib.fef_law_truncate(logits, row_len, B, K, V, ld, dt, T, k, p, m, norm, cut, cut_id, kept, status, None)

    def draw(logits=A, row_len=None, B=2, K=4, V=64, ld=64, dt=0, T=1.0, k=A, p=A, m=A, u=A, rnd=None, tok=A, conf=A, norm=A, cut=A,
             cut_id=A, kept=A, status=A):
        return lib.fef_draft_sample_truncated(logits, row_len, B, K, V, ld, dt, T, k, p, m, u, 1, 2, rnd, tok, conf, norm, cut,
                                              cut_id, kept, status, None)

    for f in (law, draw):
        assert f(dt=2) == fef.FEF_ERR_DTYPE
        for name in ("logits", "norm", "cut", "cut_id"):
            assert f(**{name: None}) == bad
        assert f(B=0) == bad and f(B=65536) == bad and f(K=0) == bad and f(K=65) == bad and f(V=0) == bad and f(ld=60) == bad
        assert f(V=fef.FEF_MAX_TRUNCATE_V + 1, ld=1 << 21) == bad
        for T in (0.0, -1.0, float("nan"), float("inf"), 1e-39):
            assert f(T=T) == bad
        assert f(logits=A + 8) == align and f(V=9, ld=10) == align and f(norm=A + 4) == align
        for name in ("row_len", "k", "p", "m", "cut", "cut_id", "kept", "status"):
            assert f(**{name: A + 2}) == align
        assert f() == fef.FEF_ERR_CUDA and f(k=None, p=None, m=None, kept=None, status=None) == fef.FEF_ERR_CUDA
    assert draw(tok=None) == bad and draw(u=A + 1) == align and draw(rnd=A + 2) == align and draw(conf=A + 2) == align
    assert draw(u=None, conf=None) == fef.FEF_ERR_CUDA

    def verify(qn=A, qc=A, qi=A, pn=A, pc=A, pi=A, T=1.0, B=2, K=4, V=64, ld=64, dt=0, ws=A, wsb=1 << 30):
        return lib.fef_spec_verify_truncated(A, A, A, qn, qc, qi, pn, pc, pi, None, B, K, V, ld, dt, T, 1, 2, None, A, A, A, ws, wsb,
                                             A, None)

    for name in ("qn", "qc", "qi", "pn", "pc", "pi"):
        assert verify(**{name: None}) == bad and verify(**{name: A + 2}) == align
    assert verify(qn=A + 4) == align and verify(pn=A + 4) == align
    assert verify(T=0.0) == bad and verify(T=float("nan")) == bad and verify(B=0) == bad and verify(K=65) == bad
    assert verify(dt=2) == fef.FEF_ERR_DTYPE and verify(ld=66) == align and verify() == fef.FEF_ERR_CUDA
    with pytest.raises(RuntimeError):
        fef.fef_law_truncate(torch.zeros(1, 1, 8), 1.0)
    with pytest.raises(RuntimeError):
        fef.fef_draft_sample_truncated(torch.zeros(1, 1, 8), 1.0)
