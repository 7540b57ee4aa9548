"""Refusals of the 8-bit cache operators that need no GPU: buffers that overlap, numbers of rows."""
import os
import re

import pytest
import torch

from test_kv8_cpu import B, P, _attn, _norm8  # noqa: F401

E = 2            # bytes of an element


# qkv of two tokens, 1024 elements each, at P; 512 elements of queries per token
@pytest.mark.parametrize("at,ld", [(0, 512), (0, 2048), (8, 1024), (512, 512), (1024, 1024), (1536, 512), (2040, 512), (-8, 512),
                                   (-1016, 512), (-512 + 8, 4096), (-4096, 4096), (-4096 + 2040, 4096)])
def test_queries_over_other_tokens_inputs_are_refused(B, at, ld):
    assert _norm8(B, q_out=P + E * at, ld=ld) == B.BS_E_ARG
    rc = B.lib().bs_op_qk_norm_rope_kv(P, P, P, 1e-6, P, P, P + E * at, ld, 2 * P, 2 * P, 64, 2, 4, 2, 128, P, 9, None, None)
    assert rc == B.BS_E_ARG


# q rows of 3584 elements
@pytest.mark.parametrize("at,ld", [(0, 4096), (8, 3584), (3584, 3584), (-8, 3584), (7160, 3584), (4096, 4096), (512 - 3584, 4096)])
def test_outputs_over_other_tokens_queries_are_refused(B, at, ld):
    assert _attn(B, out=P + E * at, q_ld=ld) == B.BS_E_ARG


OVERS = {}
for _name in ("test_write_refuses", "test_norm_refuses"):
    import test_kv8_cpu
    OVERS[_name] = getattr(test_kv8_cpu, _name).pytestmark[0].args[1]


@pytest.mark.parametrize("over", OVERS["test_write_refuses"], ids=str)
def test_write_refuses_with_queries_of_their_own(B, over):
    assert _norm8(B, **{"q_out": 4 * P, **over}) == B.BS_E_ARG


@pytest.mark.parametrize("over", OVERS["test_norm_refuses"], ids=str)
def test_norm_refuses_with_queries_of_their_own(B, over):
    a = dict(qkv=P, gq=P, gk=P, eps=1e-6, pos=P, tok_kv=P, q_out=4 * P, ld=512, kc=P, vc=P, rows=64, M=2, hq=4, hkv=2, dh=128,
             table=P, max_pos=9)
    a.update(over)
    assert B.lib().bs_op_qk_norm_rope_kv(a["qkv"], a["gq"], a["gk"], a["eps"], a["pos"], a["tok_kv"], a["q_out"], a["ld"],
                                         a["kc"], a["vc"], a["rows"], a["M"], a["hq"], a["hkv"], a["dh"], a["table"],
                                         a["max_pos"], None, None) == B.BS_E_ARG


def test_the_row_limit_is_one_number_and_named(B):
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "blockserve.h")).read()
    block, rows = map(int, re.search(r"BS_KV8_BLOCK = (\d+), BS_KV8_MAX_ROWS = (\d+)", header).groups())
    assert (B.KV8_BLOCK, B.KV8_MAX_ROWS) == (block, rows)
    q = torch.zeros(4, 256, dtype=torch.bfloat16)
    cache = B.kv8_cache(64, 2, 64, device="cpu")
    for n, why in ((rows, "CUDA"), (rows + 1, str(rows))):
        idx = torch.zeros(n + 1, dtype=torch.int32)
        with pytest.raises(B.BlockServeError, match=why):
            B.op_attention_kv8(q, *cache, idx, idx, idx, 4, scratch=torch.empty(256, dtype=torch.uint8))
    assert _attn(B, n_rows=rows + 1) == B.BS_E_ARG


def test_row_strides_beyond_31_bits_are_refused(B):
    """Passed on as they are, their low 32 bits would read other rows."""
    hq, hkv, dh, M = 4, 2, 64, 2
    far = torch.empty_strided((M, hq * dh), ((1 << 32) + hq * dh, 1), dtype=torch.bfloat16, device="meta")
    cache = B.kv8_cache(64, hkv, dh, device="cpu")
    idx = torch.zeros(M + 1, dtype=torch.int32)
    with pytest.raises(B.BlockServeError, match="row stride"):
        B.op_attention_kv8(far, *cache, idx[:2], idx, idx, hq, scratch=torch.empty(256, dtype=torch.uint8))
    qkv = torch.zeros(M, (hq + 2 * hkv) * dh, dtype=torch.bfloat16)
    kc = torch.zeros(64, hkv, dh, dtype=torch.bfloat16)
    with pytest.raises(B.BlockServeError, match="row stride"):
        B.op_qk_norm_rope_kv(qkv, None, None, 1e-6, idx, idx, kc, kc.clone(), hq, hkv, dh, B.rope_table(8, dh, 1e4, device="cpu"),
                             q_out=far)


@pytest.mark.parametrize("extra", [0, 3, 8])
def test_a_single_row_has_no_stride(B, extra):
    """One row wider than its queries by any number of elements: only the width counts."""
    q = torch.zeros(1, 256 + extra, dtype=torch.bfloat16)
    assert B._row_stride("x", -1, "q", q, 1, 256) == 256
    assert B._row_stride("x", -1, "q", torch.zeros(2, 256 + extra, dtype=torch.bfloat16), 2, 256) == 256 + extra
