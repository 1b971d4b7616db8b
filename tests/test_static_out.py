"""fef_spec_verify_static with outputs that the caller gives (the form for callers that must not allocate)."""
import builtins
import dis
import types

import pytest
import torch

import paper_2605_14305_b200 as fef


def _codes(code):
    yield code
    for c in code.co_consts:
        if isinstance(c, types.CodeType):
            yield from _codes(c)


def test_every_name_the_wrappers_use_exists():
    for name, f in vars(fef).items():
        if isinstance(f, types.FunctionType) and f.__globals__ is vars(fef):
            for code in _codes(f.__code__):
                used = {i.argval for i in dis.get_instructions(code) if i.opname == "LOAD_GLOBAL"}
                missing = {n for n in used if not hasattr(fef, n) and not hasattr(builtins, n)}
                assert not missing, (name, missing)


@pytest.mark.gpu
def test_given_outputs_equal_allocated_ones():
    fef.load(build_if_missing=True)
    B, K, V = 3, 5, 4000
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn((B, K, V), generator=g, device="cuda") * 2
    p = q + 0.5 * torch.randn((B, K, V), generator=g, device="cuda")
    tok = torch.randint(0, V, (B, K), generator=g, device="cuda", dtype=torch.int32)
    want = fef.fef_spec_verify_static(q, p, tok, 1.0, 5, 6)
    out = fef.VerifyResult(*(torch.full_like(t, 77) for t in want))
    got = fef.fef_spec_verify_static(q, p, tok, 1.0, 5, 6, out=out)
    torch.cuda.synchronize()
    assert got is out
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out.tokens.fill_(77)
    torch.cuda.synchronize()
    fef.fef_spec_verify_static(q, p, tok, 1.0, 5, 6, out=out, stream=s)
    s.synchronize()
    assert torch.equal(out.tokens, want.tokens)
