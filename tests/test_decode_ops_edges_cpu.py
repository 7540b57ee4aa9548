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


# ---- numbers of rows next to 2^31 -------------------------------------------------------------------------------

MOST = 0x7fffff00


@pytest.mark.parametrize("n", [MOST + 1, 2 ** 31 - 1])
def test_rows_whose_tiles_would_pass_31_bits_are_refused(B, n):
    far = dict(ldx=64, scale=P + 90 * G, codes=P + 40 * G)
    assert _quant(B, M=n, rows=n, **far) == B.BS_E_ARG
    wide = dict(A=P, W=P + 40 * G, C=P + 90 * G, sa=P + 300 * G, sw=P + 310 * G)
    assert _gemm(B, M=n, **wide) == B.BS_E_ARG
    assert _gemm(B, N=n, ldc=n, **wide) == B.BS_E_ARG
    rows = dict(n=n, z=P + 100 * G, out=P + 300 * G, tok=P + 500 * G, conf=P + 510 * G, row_req=P + 520 * G, row_mask=P + 530 * G)
    assert _rules(B, "rules", **rows) == B.BS_E_ARG and _rules(B, "conf", **rows) == B.BS_E_ARG


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls have made-up pointers: they must not reach a device")
def test_the_largest_numbers_of_rows_are_accepted(B):
    far = dict(ldx=64, scale=P + 90 * G, codes=P + 40 * G)
    assert _quant(B, M=MOST, rows=2 ** 31 - 1, **far) == B.BS_E_CUDA
    wide = dict(A=P, W=P + 40 * G, C=P + 90 * G, sa=P + 300 * G, sw=P + 310 * G)
    assert _gemm(B, M=MOST, **wide) == B.BS_E_CUDA
    assert _gemm(B, N=MOST, ldc=MOST, **wide) == B.BS_E_CUDA
    rows = dict(n=MOST, z=P + 100 * G, out=P + 300 * G, tok=P + 500 * G, conf=P + 510 * G, row_req=P + 520 * G, row_mask=P + 530 * G)
    assert _rules(B, "rules", **rows) == B.BS_E_CUDA and _rules(B, "conf", **rows) == B.BS_E_CUDA


@pytest.mark.parametrize("rows,ld", [(2 ** 31 - 1, 1 << 34), (2 ** 31 - 1, 1 << 33), (1 << 30, 1 << 34)])
def test_overlap_is_seen_whatever_the_strides(B, rows, ld):
    """Strides and rows that are allowed each, with an extent of up to 2^66 bytes."""
    assert _quant(B, x=P, ldx=ld, rows=rows, idx=P - 64) == B.BS_E_ARG          # the codes lie in it
    far = 1 << 60
    assert _quant(B, x=P + far, ldx=ld, rows=rows, idx=P - 64, codes=P + far + G) == B.BS_E_ARG
    n = min(rows, MOST)
    assert _gemm(B, A=P, lda=2 * ld, M=n) == B.BS_E_ARG                         # the outputs lie in A
    assert _rules(B, "rules", z=P, ld=ld, n=n, row_req=16, row_mask=16) == B.BS_E_ARG
