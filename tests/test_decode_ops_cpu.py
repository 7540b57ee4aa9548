"""8-bit row codes, 8-bit projections and logit rules without a GPU: pins of the oracle, and the refusals of the entry points
(C ABI and binding)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import decode_oracle as D


@pytest.fixture(scope="module")
def B():
    from paper_2607_08930_b200 import build
    build.build()
    from paper_2607_08930_b200 import binding
    return binding


P = 1 << 20      # stands for device pointers, far from each other: the checks come before any use
G = 1 << 33


def test_oracle_codes():
    x = np.array([[1.0, -0.5, 0.25, 127.0], [0.0, 0.0, 0.0, 0.0], [np.inf, 1.0, 0.0, 2.0]])
    _, codes, scale = D.quant(x)
    assert scale[0] == np.float32(127) * np.float32(1 / 127) and scale[1] == 2.0 ** -126 and np.isnan(scale[2])
    assert codes[0, 3] == 127 and codes[0, 0] == 1 and (codes[1:] == 0).all()
    y, codes, scale = D.quant(np.array([[3.0, 4.0]]), np.array([2.0, 1.0]), 0.0)
    assert np.allclose(y, np.array([[6.0, 4.0]]) / np.sqrt(12.5)) and codes.tolist() == [[127.0, 85.0]]


def test_oracle_rules_are_the_definition():
    z = np.array([[2.0, -2.0, 1.0, 0.5, np.nan, 3.0]], np.float32)
    y = D.rules(z, [0], 6, mask_id=5, ctx=[0, 1, 1, 5, 2], begin=[0], gen=[1], end=[5], repetition=[2.0], presence=[0.5],
                frequency=[0.25], bias_at=[0, 3], bias_tok=[2, 3, 3], bias_val=[1.0, 1.0, -4.0],
                allowed=np.array([[0b101111]], np.int32), row_mask=[0])
    # token 0 only in the prompt; 1 twice generated, 2 once with a bias; 3 two biases; 4 masked (a NaN); 5 is the mask id
    assert y.tolist() == [[1.0, -4.0 - (0.25 * 2 + 0.5), 0.5 - 0.75 + 1.0, -2.5, -np.inf, -np.inf]]
    tok, conf = D.confidence(y)
    assert tok[0] == 0 and np.isclose(conf[0], np.exp(1.0) / np.exp(y[0, :4].astype(float)).sum())
    tok, conf = D.confidence(np.array([[-np.inf, -np.inf], [np.inf, np.inf], [np.nan, 1.0], [2.0, 2.0]]))
    assert tok.tolist() == [-1, 0, 1, 0] and conf[0] == 0 and conf[1] == 0.5 and np.isnan(conf[2]) and conf[3] == 0.5


def _quant(B, **over):
    a = dict(x=P, type=0, ldx=64, idx=None, rows=4, gain=None, eps=1e-6, codes=P + G, ldc=64, scale=P + 2 * G, M=4, K=50, flag=None)
    a.update(over)
    return B.lib().bs_op_quant_i8(a["x"], a["type"], a["ldx"], a["idx"], a["rows"], a["gain"], a["eps"], a["codes"], a["ldc"],
                                  a["scale"], a["M"], a["K"], a["flag"], None)


@pytest.mark.parametrize("over", [dict(x=None), dict(x=P + 1), dict(x=P + 2, type=1), dict(type=2), dict(type=-1), dict(ldx=49),
                                  dict(ldx=1 << 40), dict(rows=3), dict(rows=0, idx=P + 3 * G), dict(idx=P + 3 * G + 2),
                                  dict(gain=P + 3 * G + 8), dict(eps=-1.0), dict(eps=float("nan")), dict(codes=None),
                                  dict(codes=P + G + 8), dict(ldc=48), dict(ldc=72), dict(scale=None), dict(scale=P + 2 * G + 2),
                                  dict(M=-1), dict(K=0), dict(K=131072, ldx=131072, ldc=131072), dict(flag=P + 1),
                                  dict(codes=P + 128), dict(scale=P), dict(scale=P + G + 64), dict(codes=P + 2 * G - 64)])
def test_row_codes_refuse(B, over):
    assert _quant(B, **over) == B.BS_E_ARG


def _gemm(B, **over):
    a = dict(A=P, lda=64, sa=P + G, W=P + 2 * G, ldw=64, sw=P + 3 * G, W2=None, sw2=None, C=P + 4 * G, ldc=30, M=4, N=30, K=50,
             mode=0, flag=None)
    a.update(over)
    return B.lib().bs_op_gemm_i8(a["A"], a["lda"], a["sa"], a["W"], a["ldw"], a["sw"], a["W2"], a["sw2"], a["C"], a["ldc"], a["M"],
                                 a["N"], a["K"], a["mode"], a["flag"], None)


@pytest.mark.parametrize("over", [dict(A=None), dict(A=P + 8), dict(lda=48), dict(lda=72), dict(sa=None), dict(sa=P + G + 1),
                                  dict(W=None), dict(W=P + 2 * G + 4), dict(ldw=49), dict(ldw=48), dict(sw=None),
                                  dict(C=None), dict(C=P + 4 * G + 4), dict(ldc=29), dict(ldc=1 << 40), dict(M=-1), dict(N=-1),
                                  dict(K=0), dict(K=131072, lda=131072, ldw=131072), dict(mode=4), dict(mode=-1), dict(mode=3),
                                  dict(mode=3, W2=P + 5 * G), dict(mode=0, W2=P + 5 * G, sw2=P + 6 * G),
                                  dict(mode=3, W2=P + 5 * G + 8, sw2=P + 6 * G), dict(C=P), dict(C=P + G), dict(C=P + 2 * G + 1024),
                                  dict(C=P + 3 * G), dict(A=P + 4 * G, C=P + 4 * G + 64), dict(flag=P + 7)])
def test_products_refuse(B, over):
    assert _gemm(B, **over) == B.BS_E_ARG


def _rules(B, call, **over):
    r = dict(vocab=100, n_reqs=4, mask_id=99, row_req=P, ctx=P + G, ctx_total=50, ctx_begin=P + 2 * G, ctx_gen=P + 3 * G,
             ctx_end=P + 4 * G, repetition=P + 5 * G, presence=P + 6 * G, frequency=P + 7 * G, bias_at=P + 8 * G, bias_tok=P + 9 * G,
             bias_val=P + 10 * G, bias_total=20, allowed=P + 11 * G, allowed_ld=4, n_masks=3, row_mask=P + 12 * G)
    a = dict(z=P + 13 * G, type=1, ld=100, out=P + 14 * G, out_ld=100, n=6, tok=P + 15 * G, conf=P + 16 * G, flag=None)
    for k, v in over.items():
        (r if k in r else a)[k] = v
    s = B.BsLogitRules(*[r[k] for k, _ in B.BsLogitRules._fields_])
    if call == "rules":
        return B.lib().bs_op_logit_rules(a["z"], a["type"], a["ld"], a["out"], a["out_ld"], a["n"], C.addressof(s), a["flag"], None)
    return B.lib().bs_op_rules_confidence(a["z"], a["type"], a["ld"], a["n"], C.addressof(s), a["tok"], a["conf"], a["flag"], None)


@pytest.mark.parametrize("call", ["rules", "conf"])
@pytest.mark.parametrize("over", [dict(z=None), dict(z=P + 13 * G + 8), dict(type=2), dict(ld=99), dict(n=-1), dict(vocab=0),
                                  dict(vocab=524289, ld=1 << 20, out_ld=1 << 20, allowed_ld=1 << 20), dict(n_reqs=-1), dict(mask_id=100),
                                  dict(mask_id=-2), dict(row_req=None), dict(row_req=P + 2), dict(ctx_total=-1),
                                  dict(ctx_total=(1 << 30) + 1), dict(ctx_begin=None), dict(ctx_gen=None), dict(ctx_end=None),
                                  dict(repetition=P + 5 * G + 1), dict(bias_total=-1), dict(bias_total=(1 << 30) + 1), dict(bias_tok=None),
                                  dict(bias_val=None), dict(allowed_ld=3), dict(n_masks=-1), dict(row_mask=None), dict(flag=P + 2)])
def test_rules_refuse(B, call, over):
    assert _rules(B, call, **over) == B.BS_E_ARG


@pytest.mark.parametrize("over", [dict(out=None), dict(out=P + 14 * G + 4), dict(out_ld=99), dict(out=P + 13 * G, out_ld=101),
                                  dict(out=P + 13 * G + 160), dict(out=P + 11 * G), dict(out=P), dict(out=P + G), dict(out=P + 10 * G)])
def test_ruled_logits_refuse(B, over):
    assert _rules(B, "rules", **over) == B.BS_E_ARG


@pytest.mark.parametrize("over", [dict(tok=None), dict(conf=None), dict(tok=P + 15 * G + 1), dict(tok=P + 13 * G), dict(conf=P + 13 * G + 64),
                                  dict(conf=P + 15 * G + 20), dict(conf=P + 11 * G), dict(tok=P)])
def test_ruled_confidence_refuses(B, over):
    assert _rules(B, "conf", **over) == B.BS_E_ARG


def test_empty_calls_are_accepted(B):
    assert _quant(B, M=0) == B.BS_OK and _gemm(B, M=0) == B.BS_OK and _gemm(B, N=0) == B.BS_OK
    assert _rules(B, "rules", n=0) == B.BS_OK and _rules(B, "conf", n=0) == B.BS_OK


def test_binding_refuses_what_is_not_on_a_gpu_or_does_not_fit(B):
    def refused(f, *a, **k):
        with pytest.raises(B.BlockServeError) as e:
            f(*a, **k)
        assert e.value.code == B.BS_E_ARG
    x = torch.zeros(3, 40)
    codes, scale = B.i8_codes(3, 40, device="cpu"), torch.ones(3)
    assert codes.stride(0) == 48
    refused(B.op_quant_i8, x)                                      # a CPU tensor
    refused(B.op_quant_i8, x.double())
    refused(B.op_quant_i8, x.t())
    refused(B.op_quant_i8, x, codes=codes[:2])
    refused(B.op_quant_i8, x, gain=torch.zeros(40))
    refused(B.op_gemm_i8, codes, scale, codes, scale)
    refused(B.op_gemm_i8, codes, scale, B.i8_codes(3, 41, device="cpu"), scale)
    refused(B.op_gemm_i8, codes, scale, codes, scale[:2])
    refused(B.op_gemm_i8, codes, scale, codes, scale, mode=1)
    refused(B.op_gemm_i8, codes, scale, codes, scale, mode=3)
    refused(B.op_gemm_i8, codes, scale, codes, scale, C_out=torch.zeros(3, 3))
    refused(B.logit_rules, 0, None, 1)
    refused(B.logit_rules, 10, None, 1, mask_id=10)
    refused(B.logit_rules, 10, None, 1, repetition=torch.ones(1))  # a penalty without a context (and on the CPU)
    rules = B.logit_rules(10, None, 2)
    refused(B.op_rules_confidence, torch.zeros(2, 10), rules)      # a CPU tensor
    refused(B.op_rules_confidence, torch.zeros(2, 11), rules)
    refused(B.op_logit_rules, torch.zeros(3, 10), rules)           # more rows than requests
    refused(B.op_logit_rules, torch.zeros(2, 10), rules, out=torch.zeros(2, 10, dtype=torch.bfloat16))
