"""Scratch that the caller gives has to be where the call runs and as large as its size says."""
import pytest
import torch

import paper_2605_14305_b200 as fef


def test_scratch_elsewhere_or_smaller_than_it_looks_is_refused():
    dev, other = torch.device("cuda", 0), torch.device("cuda", 1)

    class Given:                                             # (a tensor on a second device cannot be made everywhere)
        def __init__(self, device, contiguous=True):
            self.device, self.is_contiguous = device, lambda: contiguous

    fef._check_scratch(None, dev, "x")
    fef._check_scratch(Given(dev), dev, "x")
    for bad in (Given(other), Given(dev, False), torch.zeros(512, dtype=torch.uint8)):
        with pytest.raises(fef.FefError):
            fef._check_scratch(bad, dev, "x")
    with pytest.raises(fef.FefError):
        fef._check_scratch(torch.zeros(1, dtype=torch.uint8).expand(4096), torch.device("cpu"), "x")


@pytest.mark.gpu
def test_calls_refuse_expanded_scratch():
    fef.load(build_if_missing=True)
    B, K, V, d = 2, 4, 512, 128
    q = torch.randn((B, K, V), device="cuda")
    tok = torch.zeros((B, K), dtype=torch.int32, device="cuda")
    weight = torch.randn((V, d), device="cuda").to(torch.bfloat16)
    layer = fef.fef_lmhead_quantize(weight, 64)
    few, many, states = (torch.randn((n, d), device="cuda").to(torch.bfloat16) for n in (4, 40, B * K))
    calls = [lambda ws: fef.fef_spec_verify(q, q, tok, 1.0, 1, 1, workspace=ws),
             lambda ws: fef.fef_draft_sample(q, 1.0, 1, 1, workspace=ws),
             lambda ws: fef.fef_lmhead_verify(states, states, weight, tok, 1.0, 1, 1, workspace=ws),
             lambda ws: fef.fef_logits_adjust(q, with_norm=True, workspace=ws),
             lambda ws: fef.fef_lmhead_logits_quantized(few, layer, workspace=ws),
             lambda ws: fef.fef_lmhead_logits_quantized(many, layer, workspace=ws)]
    real = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")
    for call in calls:
        with pytest.raises(fef.FefError):
            call(torch.zeros(1, dtype=torch.uint8, device="cuda").expand(1 << 24))
        call(real)
    torch.cuda.synchronize()
