"""Calls at the borders of what the 8-bit cache operators take, against the 64-bit oracle (needs a B200)."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import kv8_oracle as K
from test_kv8_gpu import (B, EPS, HALF_BF16, THETA, attn_bound, attn_inputs, bf16, chain_tol, check_attention, host, ints,  # noqa: F401
                          prefix, random_cache, slabs, to_gpu)

pytestmark = pytest.mark.gpu


# ---- queries far from one ------------------------------------------------------------------------------------

def check_winners(got, q, hq, dh, k, v):
    """Scores so far apart that the softmax is its largest key's alone: the output is that key's V (which bf16 holds
    exactly), off by the weight's fp16 rounding in the product (2^-11) and half a bf16 step.  Query rows whose two largest
    scores lie within twice the scores' error (sums of dh products in fp32, a query element held to 2^-17 of its row's
    largest) plus 40 are left out: they are few."""
    n, g, seen = len(q), hq // k.shape[1], 0
    for h in range(hq):
        z = q[:, h] @ k[:, h // g].T / np.sqrt(dh)
        err = (np.abs(q[:, h]) @ np.abs(k[:, h // g]).T).max(1) / np.sqrt(dh) * (dh + 4) * 2.0 ** -23 + \
            np.abs(q[:, h]).max(1) * np.abs(k[:, h // g]).sum(1).max() / np.sqrt(dh) * 2.0 ** -17
        top = np.sort(z, 1)
        clear = top[:, -1] - top[:, -2] > 2 * err + 40
        want = v[z.argmax(1), h // g]
        tol = np.abs(want) * (HALF_BF16 + 2.0 ** -11 + 2.0 ** -20) + np.abs(v).max() * 2.0 ** -40
        assert (np.abs(got[:, h] - want)[clear] <= tol[clear]).all(), h
        seen += int(clear.sum())
    assert seen >= 0.8 * n * hq


@pytest.mark.parametrize("power", [24, 30, 33, 36, 45, 60, 102, 110, 116, 125])
@pytest.mark.parametrize("hq,hkv,dh,rows", [(28, 4, 128, [(1, 300)]), (32, 32, 128, [(32, 129)] * 3), (8, 2, 64, [(12, 200)]),
                                            (14, 2, 128, [(40, 200), (40, 1100)]), (8, 2, 64, [(64, 333)]),
                                            (28, 4, 128, [(300, 500)] * 6)])
def test_queries_of_any_finite_size(B, hq, hkv, dh, rows, power):
    """Every other token's queries are 2^power as large, up to the type's last binade; the others keep their results."""
    rng = np.random.default_rng(power)
    n, vis, base, kc, vc, q = attn_inputs(rng, hq, hkv, dh, rows)
    kc[1][np.isfinite(kc[1])] = 2.0 ** -20
    q = bf16(np.clip(host(q), -7.9, 7.9))                  # 7.9 x 2^125 is below the largest bf16
    q[::2] = (q[::2].double() * 2.0 ** power).to(torch.bfloat16)
    assert torch.isfinite(q).all()
    (k8, ks), (v8, vs) = to_gpu(*kc), to_gpu(*vc)
    out = host(B.op_attention_kv8(q.cuda(), k8, v8, ks, vs, ints(prefix(n)), ints(base), ints(vis), hq, max_nq=int(n.max()),
                                  max_vis=int(vis.max())))
    cu = prefix(n)
    for i in range(len(n)):
        k, v = K.span(*kc, base[i], 0, vis[i]), K.span(*vc, base[i], 0, vis[i])
        t = np.arange(cu[i], cu[i + 1])
        large, small = t[t % 2 == 0], t[t % 2 == 1]
        check_winners(out[large].reshape(-1, hq, dh), host(q[large]).reshape(-1, hq, dh), hq, dh, k, v)
        if len(small):
            ref, mag, dot, flat = K.attention(host(q[small]).reshape(-1, hq, dh), k, v)
            assert (np.abs(out[small].reshape(-1, hq, dh) - ref) <= attn_bound(ref, mag, dot, flat, np.abs(v).max(), vis[i], dh)).all()


@pytest.mark.parametrize("hq,hkv,dh,nq", [(28, 4, 128, 1), (32, 32, 128, 32), (8, 2, 64, 12), (14, 2, 128, 64), (8, 2, 64, 64)])
def test_scores_a_few_of_their_own_steps_apart(B, hq, hkv, dh, nq):
    """Keys whose scores, 2^23 to 2^30 in log2 units, differ by a few of fp32's steps there: which of them win is a matter of
    rounding, but every output is a mean of the values, between 1 and 2."""
    rng = np.random.default_rng(nq + hq)
    vis, blocks = 400, 13
    codes = np.zeros((blocks, hkv, 32, dh), np.uint8)
    codes[..., 1:17] = rng.integers(0, 16, codes[..., 1:17].shape)
    codes[..., 0] = 126                                    # 448
    values = rng.integers(56, 65, codes.shape).astype(np.uint8)      # 1 to 2
    q = np.zeros((nq, hq, dh))
    q[..., 0] = 2.0 ** rng.integers(18, 25, (nq, hq))
    q[..., 1:17] = rng.normal(size=(nq, hq, 16)) * q[..., :1] * 2.0 ** rng.integers(-10, -4, (nq, hq, 1))
    q = bf16(q.reshape(nq, hq * dh))
    (k8, ks), (v8, vs) = to_gpu(codes, np.ones((blocks, hkv))), to_gpu(values, np.ones((blocks, hkv)))
    for max_vis in (vis, 0):
        out = host(B.op_attention_kv8(q.cuda(), k8, v8, ks, vs, ints([0, nq]), ints([0]), ints([vis]), hq, max_nq=nq, max_vis=max_vis))
        assert np.isfinite(out).all() and out.min() >= 1 - 2.0 ** -8 and out.max() <= 2 * (1 + 2.0 ** -8)


@pytest.mark.parametrize("nq", [1, 64])
def test_large_queries_beside_small_ones_and_far_scales(B, nq):
    """(2^110, 2^104) against the keys (1, 0) and (0, 4): the first wins.  Scores beyond fp32 to the negative side are keys
    without weight, and a zero code meets a query and a scale whose product is beyond fp32 as a zero."""
    hq, hkv, dh = 4, 1, 128
    codes = np.zeros((3, 1, 32, dh), np.uint8)
    one, four = K.encode(np.array([1.0, 4.0]))
    codes[0, 0, 0, 0], codes[0, 0, 1, 1] = one, four
    codes[1, 0, :, 2], codes[1, 0, 5, 2] = one + 128, 0    # block 1: -1, and 0 at key 37
    vcodes = np.zeros((3, 1, 32, dh), np.uint8)
    vals = np.arange(1, 97) % 29 + 1.0
    vcodes[:, 0] = K.encode(np.floor(vals)).reshape(3, 32, 1)
    scales = np.ones((3, 1))
    q = torch.zeros(nq, hq * dh, dtype=torch.bfloat16)
    q[0, 0], q[0, 1] = 2.0 ** 110, 2.0 ** 104              # head 0: key 0
    q[0, dh + 2] = 2.0 ** 120                              # head 1: block 1 loses but for its zero
    (k8, ks), (v8, vs) = to_gpu(codes, scales), to_gpu(vcodes, np.ones((3, 1)))
    ks[1] = 2.0 ** 30                                      # head 1's products there: -2^150 and 0
    v = K.decode(vcodes)[:, 0, :, 0].reshape(-1)
    out = host(B.op_attention_kv8(q.cuda(), k8, v8, ks, vs, ints([0, nq]), ints([0]), ints([70]), hq, max_nq=nq, max_vis=0))
    out = out.reshape(nq, hq, dh)
    tol = lambda x: x * (HALF_BF16 + 2.0 ** -10)           # noqa: E731
    assert (np.abs(out[0, 0] - v[0]) <= tol(v[0])).all()
    tied = np.r_[0:32, 37, 64:70]                          # all of them score zero
    assert (np.abs(out[0, 1] - v[tied].mean()) <= tol(v[tied].mean())).all()
    assert (np.abs(out[0, 2:] - v[:70].mean()) <= tol(v[:70].mean())).all()


@pytest.mark.parametrize("hq,hkv,dh,rows", [(28, 4, 128, [(1, 77)]), (14, 2, 128, [(40, 97), (40, 130)]), (8, 2, 64, [(64, 200)]),
                                            (28, 4, 128, [(300, 330)] * 6)])
def test_queries_of_next_to_nothing_average(B, hq, hkv, dh, rows):
    """Zero query rows, and rows of 2^-120, over blocks of zeros (whose scale is the least, 2^-40) that end inside a tile."""
    rng = np.random.default_rng(len(rows) + dh)
    n, vis, base, kc, vc, q = attn_inputs(rng, hq, hkv, dh, rows)
    kc[0][kc[0] != 127] = 0
    kc[1][np.isfinite(kc[1])] = 2.0 ** -40
    q[::3] = 0
    q[1::3] = (q[1::3].double() * 2.0 ** -120).to(torch.bfloat16)
    (k8, ks), (v8, vs) = to_gpu(*kc), to_gpu(*vc)
    out = B.op_attention_kv8(q.cuda(), k8, v8, ks, vs, ints(prefix(n)), ints(base), ints(vis), hq, max_nq=int(n.max()),
                             max_vis=0)
    check_attention(host(out), q, hq, dh, n, vis, base, kc, vc)


# ---- many rows, missing hints --------------------------------------------------------------------------------

def ms_of(fn):
    for _ in range(3):
        fn()
    best = 1e9
    for _ in range(7):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        fn()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


@pytest.mark.parametrize("hq,hkv,dh,n_rows,nq", [(32, 32, 64, 512, 16), (16, 1, 128, 300, 40)])
def test_many_short_rows_without_a_query_hint(B, hq, hkv, dh, n_rows, nq):
    """Work grows with the tokens, not with rows x tokens: without max_nq a call takes at most three times as long."""
    rng = np.random.default_rng(n_rows)
    rows = [(int(a), int(b)) for a, b in zip(rng.integers(1, nq + 1, n_rows), rng.integers(0, 65, n_rows))]
    n, vis, base, kc, vc, q = attn_inputs(rng, hq, hkv, dh, rows)
    (k8, ks), (v8, vs) = to_gpu(*kc), to_gpu(*vc)
    a = (q.cuda(), k8, v8, ks, vs, ints(prefix(n)), ints(base), ints(vis), hq)
    told, untold = (lambda m=m: B.op_attention_kv8(*a, max_nq=m, max_vis=64) for m in (nq, 0))
    check_attention(host(untold()), q, hq, dh, n, vis, base, kc, vc)
    assert ms_of(untold) <= 3 * ms_of(told) + 0.02


@pytest.mark.parametrize("hq,hkv,dh,nq,top,hint", [(28, 4, 128, 1, 300, 300), (4, 2, 64, 2, 700, 0), (14, 2, 128, 10, 200, 200)])
def test_as_many_rows_as_a_call_takes(B, hq, hkv, dh, nq, top, hint):
    rng = np.random.default_rng(top)
    rows = [(int(a), int(b)) for a, b in zip(rng.integers(0, nq + 1, 1024), rng.integers(0, top + 1, 1024))]
    n, vis, base, kc, vc, q = attn_inputs(rng, hq, hkv, dh, rows)
    (k8, ks), (v8, vs) = to_gpu(*kc), to_gpu(*vc)
    out = B.op_attention_kv8(q.cuda(), k8, v8, ks, vs, ints(prefix(n)), ints(base), ints(vis), hq, max_nq=nq, max_vis=hint)
    check_attention(host(out), q, hq, dh, n, vis, base, kc, vc)


def test_write_and_read_of_many_rows(B):
    """More rows than two rounds of the search over them reach: writes bit for bit (V), and read back."""
    hq, hkv, dh = 2, 1, 64
    rng = np.random.default_rng(9)
    n, at = rng.integers(0, 4, 1500), rng.integers(0, 70, 1500)
    base, blocks = slabs(rng, at + n, gap=False)
    M, cu = int(n.sum()), prefix(n)
    qkv = bf16(rng.normal(size=(M, 4 * dh)))
    row = np.repeat(np.arange(1500), n)
    pos = at[row] + np.arange(M) - cu[row]
    cv, sv = random_cache(rng, blocks, hkv, dh)
    (k8, ks), (v8, vs) = to_gpu(*random_cache(rng, blocks, hkv, dh)), to_gpu(cv, sv)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = B.op_qk_norm_rope_kv8(qkv.cuda(), None, None, EPS, ints(pos), ints(cu), ints(base), ints(at), ints(at), k8, v8, ks, vs,
                              hq, hkv, dh, B.rope_table(100, dh, THETA), error_flag=flag)
    x = host(qkv).reshape(M, 4, dh)
    ref = K.norm_rope(x[:, :hq], None, EPS, pos, THETA)
    assert (np.abs(host(q).reshape(M, hq, dh) - ref) <= np.abs(ref) * HALF_BF16 + 2 * chain_tol(ref, dh)).all()
    rv, rsv = K.write(cv, sv, list(zip(cu[:-1], n, base, at, at)), x[:, 3:])
    assert (vs.cpu().numpy() == rsv).all() and (v8.view(torch.uint8).cpu().numpy() == rv).all()
    _, vo = B.op_kv8_read(k8, v8, ks, vs, ints(cu), ints(base), ints(at), M, error_flag=flag)
    assert (host(vo) == np.concatenate([K.span(rv, rsv, base[i], at[i], n[i]) for i in range(1500)])).all()
    assert int(flag.item()) == 0


# ---- indices that do not fit ---------------------------------------------------------------------------------

@pytest.mark.parametrize("many", [0, 33, 250])
def test_write_skips_the_queries_of_rows_that_do_not_fit(B, many):
    """A row whose span does not fit is skipped whole, as a token with a bad cache row of the bf16 cache is: its queries stay
    as they were, in place too, so that the call can be made again."""
    hq, hkv, dh = 4, 2, 64
    rng = np.random.default_rng(3)
    n = np.array([2, 1, 3, 1, 2, 1, 0, 5])
    base = np.array([16, -32, 128, 64, 0, 32, 7, 0])       # rows 0, 1, 2, 3, 4 do not fit (row 6 has no token)
    at = np.array([0, 0, 0, 64, -1, 2, 0, 20])
    bad = np.array([True] * 5 + [False] * 3)
    if many:                                               # more rows than a CTA looks up at once, long stretches of empty ones
        n = np.where(rng.random(many) < 0.5, 0, rng.integers(1, 4, many))
        n[10:many // 3] = 0
        bad = rng.random(many) < 0.3
        base = 32 * np.arange(many)
        at = np.where(bad, 32 * many, rng.integers(0, 29, many))
    M, cu = int(n.sum()), prefix(n)
    pad = 2
    qkv = bf16(rng.normal(size=(M + pad, (hq + 2 * hkv) * dh)))
    table = B.rope_table(50, dh, THETA)
    pos = np.r_[np.arange(M) % 50, 3, 3]
    (k8, ks), (v8, vs) = to_gpu(*random_cache(rng, max(4, many), hkv, dh)), to_gpu(*random_cache(rng, max(4, many), hkv, dh))
    want = K.norm_rope(host(qkv)[:, :hq * dh].reshape(-1, hq, dh), None, EPS, pos, THETA).reshape(-1, hq * dh)
    skipped = np.r_[np.repeat(bad, n), True, True]
    for inplace in (False, True):
        flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        x = qkv.cuda()
        q_out = x if inplace else torch.full((M + pad, hq * dh), 9.0, dtype=torch.bfloat16, device="cuda")
        before = host(q_out)
        B.op_qk_norm_rope_kv8(x, None, None, EPS, ints(pos), ints(cu), ints(base), ints(at), ints(at), k8, v8, ks, vs, hq, hkv, dh,
                              table, q_out=q_out, error_flag=flag)
        assert int(flag.item()) >= 100
        got = host(q_out)
        assert (got[skipped] == before[skipped]).all()
        g, w = got[~skipped, :hq * dh], want[~skipped]
        assert (np.abs(g - w).reshape(-1, hq, dh) <= (np.abs(w) * HALF_BF16).reshape(-1, hq, dh) + 2 * chain_tol(w.reshape(-1, hq, dh), dh)).all()


# ---- waits that run out --------------------------------------------------------------------------------------

@pytest.fixture()
def debug_lib(B, monkeypatch):
    from paper_2607_08930_b200 import build
    path = build.build(debug=True)
    regular = B.lib()
    monkeypatch.setattr(B, "LIB_PATH", path)
    monkeypatch.setattr(B, "_lib", None)
    assert B.lib() is not regular
    return B


@pytest.mark.parametrize("after", [0, 1, 2])
@pytest.mark.parametrize("hq,hkv,dh,rows,alone", [
    (14, 1, 128, [(9, 300)], True),                        # one CTA: everything it has is lost
    (8, 1, 64, [(16, 290)], True),
    (14, 1, 128, [(9, 1400)], False),                      # one tile of queries, its keys in chunks
    (14, 2, 128, [(40, 300), (30, 0), (40, 700)], False),
    (28, 4, 128, [(300, 500)] * 6, False)])                # two query tiles a CTA
def test_a_wait_that_runs_out_leaves_no_result(debug_lib, hq, hkv, dh, rows, alone, after):
    """In the bounds-checked build the waits of a CTA run out at key tile t when the flag holds -1 - t (the first one raises
    it, so later CTAs may go on): the flag says so, outputs are NaN or right, rows without keys zeros, and the next call is
    right."""
    rng = np.random.default_rng(len(rows) + dh)
    n, vis, base, kc, vc, q = attn_inputs(rng, hq, hkv, dh, rows)
    (k8, ks), (v8, vs) = to_gpu(*kc), to_gpu(*vc)
    flag = torch.full((1,), -1 - after, dtype=torch.int32, device="cuda")
    run = lambda: host(debug_lib.op_attention_kv8(q.cuda(), k8, v8, ks, vs, ints(prefix(n)), ints(base), ints(vis), hq,   # noqa: E731
                                                  max_nq=int(n.max()), max_vis=int(vis.max()), error_flag=flag))
    got = run()
    assert int(flag.item()) == 1
    flag.zero_()
    want = run()
    assert int(flag.item()) == 0
    check_attention(want, q, hq, dh, n, vis, base, kc, vc)
    lost = np.isnan(got)
    assert lost.any() and (got[~lost] == want[~lost]).all()
    assert not lost[np.repeat(vis == 0, n)].any()
    assert lost.all() or not alone


# ---- buffers that share memory -------------------------------------------------------------------------------

@pytest.mark.parametrize("hq,hkv,dh,rows,told", [
    (28, 4, 128, [(1, 300), (1, 0), (1, 77)], True), (28, 4, 128, [(1, 3000), (1, 20)], False), (32, 32, 128, [(32, 200)] * 9, True),
    (14, 2, 128, [(40, 300), (9, 0), (64, 90)], True), (28, 4, 128, [(300, 500)] * 6, True), (14, 1, 128, [(9, 1400)], True)])
def test_attention_in_place(B, hq, hkv, dh, rows, told):
    rng = np.random.default_rng(len(rows))
    n, vis, base, kc, vc, q = attn_inputs(rng, hq, hkv, dh, rows)
    (k8, ks), (v8, vs) = to_gpu(*kc), to_gpu(*vc)
    a = (k8, v8, ks, vs, ints(prefix(n)), ints(base), ints(vis), hq)
    kw = dict(max_nq=int(n.max()), max_vis=int(vis.max()) if told else 0)
    want = B.op_attention_kv8(q.cuda(), *a, **kw)
    x = q.cuda()
    assert B.op_attention_kv8(x, *a, out=x, **kw) is x and torch.equal(x, want)


def test_buffers_side_by_side_in_one_allocation(B):
    """Queries right before and right behind their inputs, and two rows of them around the inputs, are no overlap."""
    hq, hkv, dh, M = 4, 2, 64, 2
    width, wq = (hq + 2 * hkv) * dh, hq * dh
    rng = np.random.default_rng(1)
    qkv = bf16(rng.normal(size=(M, width)))
    table = B.rope_table(8, dh, THETA)
    mem = torch.empty(4 * M * width, dtype=torch.bfloat16, device="cuda")
    x = mem[M * width:2 * M * width].view(M, width)
    kc = torch.zeros(8, hkv, dh, dtype=torch.bfloat16, device="cuda")
    call = lambda q: B.op_qk_norm_rope_kv(x, None, None, EPS, ints([3, 4]), ints([0, 1]), kc, torch.zeros_like(kc), hq, hkv, dh,   # noqa: E731
                                          table, q_out=q)
    x.copy_(qkv)
    want = call(None)
    for q in (mem[M * width - M * wq:M * width].view(M, wq), mem[2 * M * width:2 * M * width + M * wq].view(M, wq),
              mem.as_strided((M, wq), (M * width + wq, 1), M * width - wq)):
        assert torch.equal(call(q), want) and torch.equal(x.cpu(), qkv)
    with pytest.raises(B.BlockServeError):
        call(mem.as_strided((M, wq), (M * width + wq - 8, 1), M * width - wq))
    k8, v8, ks, vs = B.kv8_cache(32, hkv, dh)
    with pytest.raises(B.BlockServeError):
        B.op_qk_norm_rope_kv8(x, None, None, EPS, ints([3, 4]), ints([0, 2]), ints([0]), ints([0]), ints([0]), k8, v8, ks, vs, hq, hkv,
                              dh, table, q_out=x[:, dh:])


# ---- small caches, tight bounds, first calls -----------------------------------------------------------------

@pytest.mark.parametrize("blocks", [1, 2, 3, 4])
@pytest.mark.parametrize("hq,hkv,dh,nq", [(14, 2, 128, 40), (8, 2, 64, 64), (28, 4, 128, 1)])
def test_caches_of_less_than_a_key_tile(B, hq, hkv, dh, nq, blocks):
    rng = np.random.default_rng(blocks)
    vis = blocks * 32 - 5
    ck, sk = random_cache(rng, blocks, hkv, dh, spread=0)
    cv, sv = random_cache(rng, blocks, hkv, dh)
    ck[-1, :, 27:], cv[-1, :, 27:] = 127, 127
    q = bf16(rng.normal(size=(nq, hq * dh)))
    (k8, ks), (v8, vs) = to_gpu(ck, sk), to_gpu(cv, sv)
    out = B.op_attention_kv8(q.cuda(), k8, v8, ks, vs, ints([0, nq]), ints([0]), ints([vis]), hq, max_nq=nq)
    check_attention(host(out), q, hq, dh, np.array([nq]), np.array([vis]), np.array([0]), (ck, sk), (cv, sv))


@pytest.mark.parametrize("hq,hkv,dh,nq,vis", [(28, 4, 128, 1, 500), (28, 4, 128, 1, 3000), (32, 32, 128, 32, 300), (8, 2, 64, 12, 400)])
def test_streamed_queries_keep_their_small_elements(B, hq, hkv, dh, nq, vis):
    """One channel of the queries is 2^12 times the others and meets keys of zero there.  The streaming kernel holds a query
    in fp16 after its row's largest element has come to [1, 2): an element is off by 2^-25 of that one at most (bf16's 8
    bits fit fp16's 11; half its least step is 2^-25), so the bound has that in place of the two-term 2^-17."""
    rng = np.random.default_rng(nq + vis)
    n, at, base, kc, vc, q = attn_inputs(rng, hq, hkv, dh, [(nq, vis)])
    q = q.reshape(nq, hq, dh)
    q[:, :, 7] = 2.0 ** 12
    q = q.reshape(nq, hq * dh)
    seen = kc[0] != 127
    kc[0][..., 7] = np.where(seen[..., 7], 0, 127)
    (k8, ks), (v8, vs) = to_gpu(*kc), to_gpu(*vc)
    out = B.op_attention_kv8(q.cuda(), k8, v8, ks, vs, ints([0, nq]), ints(base), ints([vis]), hq, max_nq=nq, max_vis=vis)
    k, v = K.span(*kc, base[0], 0, vis), K.span(*vc, base[0], 0, vis)
    ref, mag, dot, flat = K.attention(host(q).reshape(nq, hq, dh), k, v)
    tol = attn_bound(ref, mag, dot, flat * 2.0 ** -8, np.abs(v).max(), vis, dh)
    assert (np.abs(host(out).reshape(nq, hq, dh) - ref) <= tol).all()


FIRST_CALL = """
import sys, torch
from paper_2607_08930_b200 import binding as B
hq, hkv, dh, nq = 14, 2, 128, int(sys.argv[1])
torch.manual_seed(0)
ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
k8, v8, ks, vs = B.kv8_cache(2048, hkv, dh)
qkv = torch.randn(2 * nq, (hq + 2 * hkv) * dh, device="cuda").bfloat16()
idx = ints(0, nq, 2 * nq), ints(0, 1024), ints(0, 0), ints(0, 0)
pos, vis = torch.arange(2 * nq, dtype=torch.int32, device="cuda") % nq, ints(nq, nq)
table = B.rope_table(nq, dh, 1e4)
def step():
    q = B.op_qk_norm_rope_kv8(qkv, None, None, 1e-6, pos, *idx, k8, v8, ks, vs, hq, hkv, dh, table)
    return B.op_attention_kv8(q, k8, v8, ks, vs, idx[0], idx[1], vis, hq), B.op_kv8_read(k8, v8, ks, vs, idx[0], idx[1], idx[2], 2 * nq)[1]
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    got = step()
g.replay()
torch.cuda.synchronize()
want = step()
assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.isfinite(got[0].float()).all()
print("same")
"""


@pytest.mark.parametrize("nq", ["1", "70"])
def test_the_first_call_of_a_process_may_be_captured(B, nq):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALL, nq], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]
