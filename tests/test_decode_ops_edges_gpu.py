"""What the 8-bit row codes, the 8-bit projections and the logit rules do at the edges of what they accept, against the
64-bit oracle (needs a B200)."""
import itertools
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import decode_oracle as D
from test_decode_ops_gpu import B, CONF_TOL, HALF_F32, check_rules, f32, host, ints, random_codes  # noqa: F401

pytestmark = pytest.mark.gpu


def new_flag():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


# ---- bias lists that do not ascend, or name what is no token ----------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,pad", [(700, 0), (701, 0), (40001, 0), (126464, 64)])
@pytest.mark.parametrize("tok", [[5, 4], [7, 3, 9], [2, 1 << 20, 5], [600, 5, 600, 5], [-1, 3], [3, 3, 2, 2], [9, 8, 7, 6]])
def test_biases_out_of_order_touch_nothing_else(B, dtype, vocab, pad, tok):
    """The request's rows lie in the middle of a larger buffer.  Of its biases some count (which is not defined); every
    other entry, the other requests' rows and the memory around them are as without the list."""
    rng = np.random.default_rng(vocab + len(tok))
    rows, mid = 5, [1, 2, 3]
    row_req = np.array([0, 1, 1, 1, 2])
    ctx = rng.integers(0, vocab, 60)
    ctx[:3] = [3, 5, 600]
    r = dict(mask_id=vocab - 1, ctx=ctx, begin=[0, 0, 20], gen=[5, 9, 30], end=[20, 20, 60],
             repetition=np.array([1.2, 1.3, 1.1], np.float32), presence=np.array([0.3, 0.2, 0.1], np.float32))
    val = np.linspace(0.5, 2.0, len(tok)).astype(np.float32)
    z = torch.from_numpy((3 * rng.normal(size=(rows, vocab))).astype(np.float32)).to(dtype)
    plain = D.rules(z.float().numpy(), row_req, vocab, **r)
    rules = B.logit_rules(vocab, ints(row_req), 3, mask_id=vocab - 1, ctx=ints(ctx), ctx_begin=ints(r["begin"]),
                          ctx_gen=ints(r["gen"]), ctx_end=ints(r["end"]), repetition=f32(r["repetition"]),
                          presence=f32(r["presence"]), bias_at=ints([0, 0, len(tok), len(tok)]), bias_tok=ints(tok),
                          bias_val=f32(val))
    named = sorted({t for t in tok if 0 <= t < vocab - 1})
    rest = np.setdiff1d(np.arange(vocab), named)
    guard = 16                                               # rows of it on either side

    def buffer():
        store = torch.full((rows + 2 * guard, vocab + pad), 77.0, dtype=dtype, device="cuda")
        return store, store[guard:guard + rows, :vocab]

    def check(store, view):
        got, want = view.cpu(), torch.from_numpy(plain).to(dtype)
        assert torch.equal(got[[0, 4]], want[[0, 4]])
        assert torch.equal(got[:, rest], want[:, rest])
        view.fill_(77.0)
        assert (store == 77.0).all()

    store, view = buffer()
    view.copy_(z.cuda())
    flag = new_flag()
    tok_out, conf = torch.full((rows + 8,), -9, dtype=torch.int32, device="cuda"), torch.full((rows + 8,), -9.0, device="cuda")
    B.op_rules_confidence(view, rules, tok=tok_out[4:4 + rows], conf=conf[4:4 + rows], error_flag=flag)
    assert int(flag) >= 100
    assert (tok_out[[0, 1, 2, 3, -1]] == -9).all() and (conf[[0, 1, 2, 3, -1]] == -9).all()
    # the outcomes that some of the biases could give
    some = [D.confidence(plain)]
    for n in range(1, len(tok) + 1):
        for which in itertools.combinations([i for i, t in enumerate(tok) if t in named], n):
            y = plain.copy()
            for i in which:
                y[mid, tok[i]] += val[i]
            some.append(D.confidence(y))
    t, c = tok_out[4:4 + rows].cpu().numpy(), host(conf[4:4 + rows])
    for row in range(rows):
        assert any(t[row] == tt[row] and abs(c[row] - cc[row]) <= cc[row] * CONF_TOL for tt, cc in some), row
    flag.zero_()
    out_store, out = buffer()
    B.op_logit_rules(view, rules, out=out, error_flag=flag)
    assert int(flag) >= 100
    check(out_store, out)
    flag.zero_()
    B.op_logit_rules(view, rules, error_flag=flag)           # in place
    assert int(flag) >= 100
    check(store, view)


@pytest.mark.parametrize("vocab,length", [(2003, 300), (9000, 9000), (40001, 30000)])
def test_long_lists_of_biases_in_any_order(B, vocab, length):
    rng = np.random.default_rng(length)
    tok = rng.integers(-5, vocab // 2, length)               # the upper half is not named
    store = torch.full((24, vocab), 77.0, device="cuda")
    z = torch.randn(4, vocab, device="cuda")
    store[12:16] = z
    flag = new_flag()
    rules = B.logit_rules(vocab, None, 4, bias_at=ints([0, 0, length, length, length]), bias_tok=ints(tok),
                          bias_val=torch.ones(length, device="cuda"))
    _, conf = B.op_rules_confidence(store[12:16].clone(), rules)
    B.op_logit_rules(store[12:16], rules, error_flag=flag)
    assert int(flag) >= 100 and torch.isfinite(conf).all()
    assert torch.equal(store[12:16][[0, 2, 3]], z[[0, 2, 3]])
    rest = np.setdiff1d(np.arange(vocab), tok)
    assert torch.equal(store[13, rest], z[1, rest]) and torch.isfinite(store[13]).all()
    assert (store[:12] == 77.0).all() and (store[16:] == 77.0).all()


# ---- zeros of both signs ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,pad", [(1000, 0), (1001, 2), (40001, 0), (126464, 0)])
@pytest.mark.parametrize("masked", [False, True])
def test_the_lowest_of_zeros_of_both_signs(B, dtype, vocab, pad, masked):
    """Rows whose largest logits are a zero of one sign and, in another warp's entries, a zero of the other: the lower id
    every time, whichever warp is first."""
    rng = np.random.default_rng(vocab)
    rows = 256
    z = np.full((rows, vocab), -4.0, np.float32)
    low = rng.integers(0, vocab - 300, rows)
    high = low + rng.integers(100, np.minimum(vocab - low, 5000))
    z[np.arange(rows), low] = np.where(np.arange(rows) % 4 < 3, -0.0, 0.0)
    z[np.arange(rows), high] = np.where(np.arange(rows) % 4 < 3, 0.0, -0.0)
    store = torch.zeros(rows, vocab + pad, dtype=dtype, device="cuda")
    store[:, :vocab] = f32(z).to(dtype)
    every = torch.full((1, (vocab + 31) // 32), -1, dtype=torch.int32, device="cuda")
    # (request 0's context holds the lower zero of a few rows, which a repetition penalty keeps)
    rules = B.logit_rules(vocab, torch.zeros(rows, dtype=torch.int32, device="cuda"), 1, ctx=ints(low[:5]), ctx_begin=ints([0]),
                          ctx_gen=ints([5]), ctx_end=ints([5]), repetition=f32([1.25]), allowed=every if masked else None,
                          row_mask=torch.zeros(rows, dtype=torch.int32, device="cuda") if masked else None)
    for _ in range(30):
        tok, _ = B.op_rules_confidence(store[:, :vocab], rules)
        assert np.array_equal(tok.cpu().numpy(), low)


# ---- members of rules that are absent ---------------------------------------------------------------------------

@pytest.mark.parametrize("left", [dict(n_masks=-5), dict(ctx_total=-1), dict(bias_total=-(1 << 40)), dict(allowed_ld=-3),
                                  dict(ctx_total=1 << 50, bias_total=1 << 50)])
def test_counts_of_absent_rules_do_not_matter(B, left):
    """What a program leaves in the counts that belong to NULL members."""
    z = torch.randn(6, 500, device="cuda")
    rules = B.logit_rules(500, None, 6, mask_id=9)
    want, want_conf = B.op_rules_confidence(z, rules)
    for k, v in left.items():
        setattr(rules.struct, k, v)
    flag = new_flag()
    tok, conf = B.op_rules_confidence(z, rules, error_flag=flag)
    assert torch.equal(tok, want) and torch.equal(conf, want_conf) and int(flag) == 0
    out = B.op_logit_rules(z, rules, out=torch.empty_like(z), error_flag=flag)
    z[:, 9] = -float("inf")
    assert torch.equal(out, z) and int(flag) == 0


def test_tensors_without_elements_are_rules_all_the_same(B):
    """A grammar of no masks, of which rows name one, and a context of no tokens, of which a request has some: both are out
    of range, not absent."""
    z = torch.randn(4, 500, device="cuda")
    words = torch.empty(0, 16, dtype=torch.int32, device="cuda")
    rules = B.logit_rules(500, None, 4, allowed=words, row_mask=ints([-1, 0, -1, 3]))
    flag = new_flag()
    tok, conf = B.op_rules_confidence(z, rules, error_flag=flag)
    assert int(flag) >= 100 and tok.tolist()[1::2] == [-1, -1] and conf.tolist()[1::2] == [0, 0]
    assert torch.equal(tok[::2].long(), z[::2].argmax(1))
    flag.zero_()
    out = torch.full_like(z, 7.0)
    B.op_logit_rules(z, rules, out=out, error_flag=flag)
    assert int(flag) >= 100 and torch.equal(out[::2], z[::2]) and (out[1::2] == 7).all()
    none, zeros = torch.empty(0, dtype=torch.int32, device="cuda"), ints([0, 0, 0, 0])
    for end, raised in ((zeros, False), (ints([0, 0, 1, 0]), True)):
        rules = B.logit_rules(500, None, 4, ctx=none, ctx_begin=zeros, ctx_gen=zeros, ctx_end=end, presence=f32([1, 1, 1, 1]))
        flag.zero_()
        assert torch.equal(B.op_logit_rules(z, rules, out=out, error_flag=flag), z) and (int(flag) >= 100) == raised


# ---- RMS norms of rows far from one -----------------------------------------------------------------------------

POWERS = [0, 126, 100, 65, 63, 61, 30, -30, -45, -49, -51, -60, -74, -80, -99, -101, -120, -133]      # of the rows


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("k,pad", [(1, 0), (9, 0), (384, 0), (385, 0), (3584, 8), (18944, 0), (40001, 0)])
@pytest.mark.parametrize("eps", [1e-5, 1e-38, 0.0])
@pytest.mark.parametrize("power", [0, 100, -60])
def test_codes_of_rms_norms_far_from_one(B, dtype, k, pad, eps, power):
    """Squares, or products with the gains, beyond what fp32 holds at either end, beside ordinary rows, rows of zeros and
    rows without a scale.  Bounds as for ordinary rows: the sum of at most 32 terms a thread (long rows: k / 1024) and ten
    joins, its root and the products, relative error below delta; a code within 127 * 2 delta of a rounded quotient."""
    rng = np.random.default_rng((k + power) % 2 ** 32)
    x = rng.uniform(0.5, 1, size=(3 * len(POWERS), k)) * rng.choice([-1, 1], size=(3 * len(POWERS), k))
    x = x * 2.0 ** np.repeat(POWERS, 3)[:, None]
    x[::7, k // 2:] *= 2.0 ** -10                             # a smaller half
    x[10] = 0.0
    x[20, 0], x[30, k - 1], x[40, 0] = np.inf, np.nan, -np.inf
    x = torch.from_numpy(x).to(dtype)
    gain = torch.from_numpy((1 + 0.2 * rng.uniform(-1, 1, size=k)) * 2.0 ** power).bfloat16()
    store = torch.zeros(x.shape[0], k + pad, dtype=dtype, device="cuda")
    store[:, :k] = x.cuda()
    got, s = B.op_quant_i8(store[:, :k], gain=gain.cuda(), eps=eps)
    with np.errstate(all="ignore"):
        e = np.float64(np.float32(eps))
        y, _, scale = D.quant(host(x), host(gain), e)
        none = ~np.isfinite(y).all(1)
    assert none[[20, 30, 40]].all() and none.sum() == 3 + (eps == 0)
    got, s = host(got), host(s)
    assert np.array_equal(np.isnan(s), none) and (got[none] == 0).all()
    y, scale, got, s = y[~none], scale[~none], got[~none], s[~none]
    delta = (max(32, k / 1024) + 10 + 8) * HALF_F32
    assert (np.abs(s - scale) <= scale * (delta + 2 * HALF_F32)).all()
    assert (np.abs(got - y / s[:, None]) <= 0.5 + 127 * 2 * delta).all()


def test_a_norm_beyond_fp32_has_no_scale(B):
    """The row's y itself is too large: 127 elements of zero and one whose y is sqrt(128) * 2^125."""
    x = torch.zeros(2, 128, device="cuda")
    x[:, 5] = 1.0
    gain = torch.ones(128, dtype=torch.bfloat16, device="cuda")
    codes, s = B.op_quant_i8(x, gain=gain * 2.0 ** 125, eps=0.0)
    assert torch.isnan(s).all() and (codes == 0).all()
    codes, s = B.op_quant_i8(x, gain=gain * 2.0 ** 123, eps=0.0)
    assert torch.isfinite(s).all() and (codes[:, 5] == 127).all() and (codes.sum(1) == 127).all()


# ---- products: each rounding, and no other ----------------------------------------------------------------------

@pytest.mark.parametrize("mode", [0, 1, 2])
@pytest.mark.parametrize("m,n,k,cpad", [(1, 130, 20000, 0), (3, 130, 33, 6), (16, 640, 9000, 0), (64, 4608, 3584, 0),
                                        (64, 128, 131071, 0), (128, 520, 6000, 3), (200, 384, 18944, 0), (256, 2048, 16384, 0),
                                        (300, 520, 777, 24), (512, 1024, 8192, 0), (512, 3584, 2000, 0), (1025, 1300, 513, 1),
                                        (3000, 2500, 300, 0)])
def test_products_have_the_stated_roundings_alone(B, mode, m, n, k, cpad):
    """The exact sum to fp32, times w_scale, times a_scale, then to bf16 or added in fp32: equal, however the call is cut."""
    rng = np.random.default_rng(m + n + k)
    a, ta = random_codes(rng, m, k)
    w, tw = random_codes(rng, n, k)
    sa, sw = rng.uniform(0.5, 2, m).astype(np.float32), (rng.uniform(0.5, 2, n) / k).astype(np.float32)
    z = (a.astype(np.float64) @ w.astype(np.float64).T).astype(np.float32) * sw * sa[:, None]
    assert z.dtype == np.float32
    out = torch.full((m, n + cpad), 3.0, dtype=torch.bfloat16 if mode == 0 else torch.float32, device="cuda")
    if mode == 1:
        base = (40 * rng.normal(size=(m, n))).astype(np.float32)
        out[:, :n] = f32(base)
        z = base + z
    B.op_gemm_i8(ta, f32(sa), tw, f32(sw), mode=mode, C_out=out[:, :n])
    assert torch.equal(out[:, :n].cpu(), torch.from_numpy(z).to(out.dtype))
    assert (out[:, n:] == 3.0).all()


# ---- launches ---------------------------------------------------------------------------------------------------

EDGES = """
import ctypes as C
import torch
from paper_2607_08930_b200 import binding as B
x, w = torch.randn(40, 256, device="cuda"), torch.randn(700, 256, device="cuda")
rules = B.logit_rules(700, None, 40, mask_id=7)
codes, wq, y = B.op_quant_i8(x), B.op_quant_i8(w), torch.randn(40, 700, device="cuda")
rt = C.CDLL("libcudart.so.12")
for op in (lambda: B.op_quant_i8(x), lambda: B.op_gemm_i8(*codes, *wq, mode=2), lambda: B.op_rules_confidence(y, rules),
           lambda: B.op_logit_rules(y, rules)):
    g = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(g):
        op(), op(), op()
    n, tail, head, data = C.c_size_t(8), (C.c_void_p * 8)(), (C.c_void_p * 8)(), (C.c_ubyte * 8 * 8)()
    assert rt.cudaGraphGetEdges_v2(C.c_void_p(g.raw_cuda_graph()), tail, head, data, C.byref(n)) == 0
    print(n.value, sum(data[i][2] == 1 for i in range(n.value)))          # (from port, to port, type, ..): 1 is programmatic
"""


@pytest.mark.parametrize("off", [False, True])
def test_the_switch_for_plain_launches(B, off):
    """Three calls in a row depend on one another, through programmatic edges unless BS_NO_PDL is set."""
    env = {k: v for k, v in os.environ.items() if k != "BS_NO_PDL"}
    if off:
        env["BS_NO_PDL"] = "1"
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", EDGES], cwd=root, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    edges = [tuple(map(int, line.split())) for line in r.stdout.splitlines()]
    assert edges == [(2, 0 if off else 2)] * 4


# ---- the largest vocabulary -------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("all_of_it", [False, True])
def test_the_largest_vocabulary(B, dtype, all_of_it):
    """Shares of 65536 entries, of which a few or all are touched; a bias for each token of one request."""
    vocab = B.RULES_MAX_VOCAB
    rng = np.random.default_rng(vocab)
    n = np.array([0, vocab + 1000 if all_of_it else 900])
    ctx = np.concatenate([rng.permutation(vocab), rng.integers(0, vocab, 1000)])[:n[1]]
    biases = np.array([vocab - 1 if all_of_it else 70, 3])
    tok = np.concatenate([np.sort(rng.permutation(vocab)[:b]) for b in biases])
    bits = rng.random((2, vocab)) < np.array([[0.5], [0.00001]])
    r = dict(row_req=np.array([0, 1, 1, -1]), mask_id=vocab - 1, ctx=ctx, begin=np.array([0, 0]), gen=np.array([0, 500]), end=n,
             repetition=np.array([1.5, 1.25], np.float32), presence=np.array([0.25, 0.5], np.float32),
             frequency=np.array([0.5, 0.125], np.float32), bias_at=np.concatenate([[0], np.cumsum(biases)]), bias_tok=tok,
             bias_val=rng.normal(size=len(tok)).astype(np.float32), row_mask=np.array([-1, 0, 1, 0]),
             allowed=np.packbits(bits, axis=1, bitorder="little").view(np.int32))
    check_rules(B, (3 * rng.normal(size=(4, vocab))).astype(np.float32), r, vocab, 2, dtype)


def test_a_list_that_keeps_one_share_busy_for_seconds(B):
    """2^25 equal biases, which one thread adds one after the other: the CTAs that join the row wait for it."""
    vocab, n = 126464, 1 << 25
    z = torch.randn(2, vocab, device="cuda")
    val = torch.ones(n, device="cuda")
    val[1::2] = -1.0
    z[:, 5] = 3.0
    rules = B.logit_rules(vocab, None, 2, bias_at=ints([0, n, n]), bias_tok=torch.full((n,), 5, dtype=torch.int32, device="cuda"),
                          bias_val=val)
    flag = new_flag()
    tok, conf = B.op_rules_confidence(z, rules, error_flag=flag)
    want, want_conf = B.op_rules_confidence(z, B.logit_rules(vocab, None, 2))
    assert int(flag) == 0 and torch.equal(tok, want)
    assert (np.abs(host(conf) - host(want_conf)) <= host(want_conf) * 2 * CONF_TOL).all()
