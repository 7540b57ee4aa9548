"""Edges of the 8-bit row codes, the 8-bit projections and the logit rules that need no GPU."""
import pytest
import torch

from test_decode_ops_cpu import B, G, P, _gemm, _quant, _rules  # noqa: F401


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls have made-up pointers: they must not reach a device")
def test_a_missing_device_is_not_an_argument_error(B):
    """So that a call that is refused without a GPU is refused for its arguments."""
    valid = [_quant(B), _quant(B, type=1), _quant(B, gain=P + 3 * G, idx=P + 4 * G, rows=1), _rules(B, "rules"), _rules(B, "conf"),
             _rules(B, "rules", out=P + 13 * G), _rules(B, "conf", row_req=None, n_reqs=6, row_mask=None, n_masks=6)]
    valid += [_gemm(B, mode=m) for m in range(3)] + [_gemm(B, mode=3, W2=P + 5 * G, sw2=P + 6 * G)]
    assert valid == [B.BS_E_CUDA] * len(valid)
