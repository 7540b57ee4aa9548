"""The 8-bit KV cache without a GPU: pins of the oracle, and the refusals of the four entry points (C ABI and binding)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import kv8_oracle as K


@pytest.fixture(scope="module")
def B():
    from paper_2607_08930_b200 import build
    build.build()
    from paper_2607_08930_b200 import binding
    return binding


def test_oracle_codes_match_the_type():
    codes = np.arange(256, dtype=np.uint8)
    ref = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(K.decode(codes), ref, equal_nan=True)
    real = codes[~np.isnan(ref)]
    assert np.array_equal(K.encode(K.decode(real)), real)                 # a code's value encodes to the code
    rng = np.random.default_rng(0)
    x = (rng.normal(size=20000) * 2.0 ** rng.integers(-9, 8, 20000)).astype(np.float32)
    x = np.concatenate([x[np.abs(x) <= 448], [0.0, 448.0, -448.0, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -7]]).astype(np.float32)
    ref = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(K.encode(x.astype(np.float64)), ref)
    assert K.encode(np.array([1e9, -np.inf, np.nan])).tolist() == [126, 254, 127]


def test_oracle_scale_is_the_smallest_power_that_holds():
    for a in (1.0, 447.9, 448.0, 448.1, 3e-5, 1e9):
        k = K.scale_exponent(a)
        assert a <= 448 * 2.0 ** k and a > 448 * 2.0 ** (k - 1)
    assert K.scale_exponent(0.0) == K.KMIN and K.scale_exponent(1e30) == K.KMAX


def test_oracle_rewrite_is_exact_unless_values_go_subnormal():
    rng = np.random.default_rng(1)
    codes = rng.integers(0, 126, (2, 1, 32, 64)).astype(np.uint8)
    scales = np.ones((2, 1))
    new = np.full((1, 1, 64), 448.0 * 8)
    c, s = K.write(codes, scales, [(0, 1, 32, 5, 20)], new)
    assert s[1, 0] == 8.0 and s[0, 0] == 1.0
    old, now = K.span(codes, scales, 32, 0, 20), K.span(c, s, 32, 0, 20)
    keep = np.arange(20) != 5
    assert np.abs(now - old)[keep].max() <= 8 * 2.0 ** -10                # half of the subnormal step at the new scale
    big = np.abs(old) >= 8 * 2.0 ** -6
    assert (now == old)[keep][big[keep]].all()
    assert (c[1, 0, 20:] == codes[1, 0, 20:]).all()                       # positions that hold nothing stay as they were


P = 1 << 20      # stands for a device pointer: the checks come before any use


def _attn(B, **over):
    a = dict(q=P, q_ld=3584, k8=P, v8=P, ks=P, vs=P, kv_rows=64, out=P, cu=P, base=P, vis=P, n_rows=2, M=2, max_nq=1,
             max_vis=10, hq=28, hkv=4, dh=128, scratch=P, nbytes=1 << 40)
    a.update(over)
    return B.lib().bs_op_attention_kv8(a["q"], a["q_ld"], a["k8"], a["v8"], a["ks"], a["vs"], a["kv_rows"], a["out"], a["cu"],
                                       a["base"], a["vis"], a["n_rows"], a["M"], a["max_nq"], a["max_vis"], a["hq"], a["hkv"],
                                       a["dh"], a["scratch"], a["nbytes"], None, None)


@pytest.mark.parametrize("over", [dict(q=None), dict(q=P + 2), dict(q_ld=3583), dict(q_ld=3588), dict(k8=None), dict(vs=P + 4),
                                  dict(kv_rows=63), dict(kv_rows=0), dict(kv_rows=1 << 31), dict(out=None), dict(cu=None),
                                  dict(base=None), dict(vis=None), dict(n_rows=-1), dict(n_rows=1025), dict(M=-1),
                                  dict(max_nq=-1), dict(max_vis=-1), dict(hq=27), dict(hkv=0), dict(hq=66, hkv=2, q_ld=66 * 128),
                                  dict(dh=96), dict(dh=0), dict(scratch=None, max_vis=0), dict(scratch=P + 16),
                                  dict(nbytes=1024, max_vis=0)])
def test_attention_refuses(B, over):
    assert _attn(B, **over) == B.BS_E_ARG


def test_empty_calls_are_accepted(B):
    assert _attn(B, M=0) == B.BS_OK and _attn(B, n_rows=0) == B.BS_OK
    L = B.lib()
    assert L.bs_op_kv8_read(None, None, None, None, 0, None, None, None, 1, 0, 4, 128, None, None, None, None) == B.BS_OK
    uses = L.bs_op_attention_kv8_uses_scratch
    assert uses(2, 2, 1, 0, 28, 4, 128) == 1 and uses(2, 2, 1, 10, 28, 4, 128) == 0 and uses(2, 64, 32, 300, 28, 4, 128) == 0
    assert uses(2, 64, 32, 40000, 28, 4, 128) == 1 and uses(2, 2, 1, 40000, 28, 4, 128) == 1 and uses(2, 2, 1, 0, 28, 5, 128) == 0
    assert L.bs_op_attention_kv8_scratch_bytes(28, 4, 128) > 0 and L.bs_op_attention_kv8_scratch_bytes(28, 5, 128) == 0


def _norm8(B, **over):
    a = dict(qkv=P, gq=P, gk=P, eps=1e-6, pos=P, cu=P, base=P, at=P, had=P, n=2, q_out=P, ld=512, k8=P, v8=P, ks=P, vs=P,
             rows=64, M=2, hq=4, hkv=2, dh=128, table=P, max_pos=9)
    a.update(over)
    return B.lib().bs_op_qk_norm_rope_kv8(a["qkv"], a["gq"], a["gk"], a["eps"], a["pos"], a["cu"], a["base"], a["at"], a["had"],
                                          a["n"], a["q_out"], a["ld"], a["k8"], a["v8"], a["ks"], a["vs"], a["rows"], a["M"],
                                          a["hq"], a["hkv"], a["dh"], a["table"], a["max_pos"], None, None)


@pytest.mark.parametrize("over", [dict(qkv=None), dict(qkv=P + 8), dict(gq=None), dict(gk=None), dict(eps=-1.0),
                                  dict(eps=float("nan")), dict(pos=None), dict(cu=None), dict(base=None), dict(at=None),
                                  dict(had=None), dict(n=-1), dict(q_out=None), dict(ld=511), dict(ld=516), dict(k8=P + 1),
                                  dict(ks=None), dict(rows=48), dict(M=-2), dict(hq=5), dict(dh=80), dict(table=None),
                                  dict(max_pos=0)])
def test_write_refuses(B, over):
    assert _norm8(B, **over) == B.BS_E_ARG


@pytest.mark.parametrize("over", [dict(qkv=None), dict(gk=None), dict(tok_kv=None), dict(kc=None), dict(vc=P + 2), dict(rows=0),
                                  dict(ld=8), dict(hq=3), dict(dh=32), dict(max_pos=-1), dict(M=-1)])
def test_norm_refuses(B, over):
    a = dict(qkv=P, gq=P, gk=P, eps=1e-6, pos=P, tok_kv=P, q_out=P, ld=512, kc=P, vc=P, rows=64, M=2, hq=4, hkv=2, dh=128,
             table=P, max_pos=9)
    a.update(over)
    assert B.lib().bs_op_qk_norm_rope_kv(a["qkv"], a["gq"], a["gk"], a["eps"], a["pos"], a["tok_kv"], a["q_out"], a["ld"],
                                         a["kc"], a["vc"], a["rows"], a["M"], a["hq"], a["hkv"], a["dh"], a["table"],
                                         a["max_pos"], None, None) == B.BS_E_ARG


@pytest.mark.parametrize("over", [dict(k8=None), dict(vs=P + 8), dict(rows=31), dict(cu=None), dict(base=None), dict(at=None),
                                  dict(n=-1), dict(total=-1), dict(hkv=0), dict(dh=100), dict(k_out=None), dict(v_out=P + 4)])
def test_read_refuses(B, over):
    a = dict(k8=P, v8=P, ks=P, vs=P, rows=64, cu=P, base=P, at=P, n=2, total=3, hkv=4, dh=64, k_out=P, v_out=P)
    a.update(over)
    assert B.lib().bs_op_kv8_read(a["k8"], a["v8"], a["ks"], a["vs"], a["rows"], a["cu"], a["base"], a["at"], a["n"],
                                  a["total"], a["hkv"], a["dh"], a["k_out"], a["v_out"], None, None) == B.BS_E_ARG


def test_rope_table_on_the_host(B):
    assert B.lib().bs_rope_table(None, 4, 64, 10000.0) == B.BS_E_ARG
    assert B.lib().bs_rope_table(P, 0, 64, 10000.0) == B.BS_E_ARG
    assert B.lib().bs_rope_table(P, 4, 63, 10000.0) == B.BS_E_ARG
    assert B.lib().bs_rope_table(P, 4, 64, 0.0) == B.BS_E_ARG
    t = B.rope_table(70, 64, 500.0, device="cpu").numpy()
    ang = np.arange(70)[:, None] * 500.0 ** (-2.0 * np.arange(32) / 64)
    assert t.shape == (70, 32, 2)
    assert np.abs(t[..., 0] - np.cos(ang)).max() < 2.0 ** -24 and np.abs(t[..., 1] - np.sin(ang)).max() < 2.0 ** -24


def test_binding_refuses_tensors_that_do_not_fit(B):
    """On the CPU: every check of the binding comes before the library is asked for anything."""
    hq, hkv, dh, M = 4, 2, 64, 3
    qkv = torch.zeros(M, (hq + 2 * hkv) * dh, dtype=torch.bfloat16)
    g = torch.ones(dh, dtype=torch.bfloat16)
    pos = torch.zeros(M, dtype=torch.int32)
    table = B.rope_table(8, dh, 1e4, device="cpu")
    cache = B.kv8_cache(70, hkv, dh, device="cpu")
    assert cache[0].shape == (3, hkv, 32, dh) and cache[2].shape == (3, hkv)
    cu, base = torch.tensor([0, 3], dtype=torch.int32), torch.zeros(1, dtype=torch.int32)

    def refused(fn, *a, **k):
        with pytest.raises(B.BlockServeError) as e:
            fn(*a, **k)
        assert e.value.code == B.BS_E_ARG
        return str(e.value)

    ok = (qkv, g, g, 1e-6, pos, cu, base, base, base, *cache, hq, hkv, dh, table)
    assert "CUDA" in refused(B.op_qk_norm_rope_kv8, *ok)                            # nothing wrong but the device
    refused(B.op_qk_norm_rope_kv8, qkv.float(), *ok[1:])
    refused(B.op_qk_norm_rope_kv8, qkv[:, :64], *ok[1:])
    refused(B.op_qk_norm_rope_kv8, qkv, None, *ok[2:])
    refused(B.op_qk_norm_rope_kv8, *ok[:4], pos.long(), *ok[5:])
    refused(B.op_qk_norm_rope_kv8, *ok[:4], pos[:2], *ok[5:])
    refused(B.op_qk_norm_rope_kv8, *ok[:6], base[:0], *ok[7:])
    refused(B.op_qk_norm_rope_kv8, *ok[:9], cache[0].view(torch.uint8), *ok[10:])
    refused(B.op_qk_norm_rope_kv8, *ok[:-1], table[:, :16].contiguous())
    refused(B.op_qk_norm_rope_kv8, *ok, q_out=torch.zeros(M, 32, dtype=torch.bfloat16))
    refused(B.op_qk_norm_rope_kv8, *ok, q_out=torch.zeros(M - 1, hq * dh, dtype=torch.bfloat16))
    refused(B.op_qk_norm_rope_kv8, *ok, error_flag=torch.zeros(1))
    kc = torch.zeros(64, hkv, dh, dtype=torch.bfloat16)
    assert "CUDA" in refused(B.op_qk_norm_rope_kv, *ok[:5], pos, kc, kc, hq, hkv, dh, table)
    refused(B.op_qk_norm_rope_kv, *ok[:5], pos, kc[:, :1], kc, hq, hkv, dh, table)
    refused(B.op_qk_norm_rope_kv, *ok[:5], pos, kc.transpose(0, 1), kc.transpose(0, 1), hq, hkv, dh, table)
    q = torch.zeros(M, hq * dh, dtype=torch.bfloat16)
    at = (q, *cache, cu, base, base, hq)
    scratch = torch.empty(256, dtype=torch.uint8)
    assert "CUDA" in refused(B.op_attention_kv8, *at, scratch=scratch)
    refused(B.op_attention_kv8, q.half(), *at[1:], scratch=scratch)
    refused(B.op_attention_kv8, q.t(), *at[1:], scratch=scratch)
    refused(B.op_attention_kv8, q, cache[0][:, :, :16], *at[2:], scratch=scratch)
    refused(B.op_attention_kv8, *at, scratch=scratch.float())
    refused(B.op_attention_kv8, *at, scratch=scratch, out=q[:1])
    assert "CUDA" in refused(B.op_kv8_read, *cache, cu, base, base, 3)
    refused(B.op_kv8_read, *cache, cu, base, base, 3, k_out=torch.zeros(2, hkv, dh, dtype=torch.bfloat16))
