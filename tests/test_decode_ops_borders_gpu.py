"""Calls at the borders of what the 8-bit projections and the logit rules take, and runs of the operators together, against
the 64-bit oracle (needs a B200)."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import decode_oracle as D
from test_decode_ops_gpu import (B, CONF_TOL, HALF_BF16, HALF_F32, check_gemm, check_rules, f32, host, ints, make_rules,  # noqa: F401
                                 random_codes, to_rules)

pytestmark = pytest.mark.gpu


def new_flag():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


# ---- what a row may hold --------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [33, 1000, 40001, 126464])
def test_odd_values_and_masks(B, dtype, vocab):
    """Rows of which nothing is left, rows of -infinity, infinities and NaN where the mask forbids them and where it does
    not, ties, and the type's lowest value as a logit."""
    rng = np.random.default_rng(vocab)
    rows, reqs = 14, 5
    r = make_rules(rng, rows, vocab, reqs, 30, 4, 3)
    words = (vocab + 31) // 32
    bits = np.zeros((3, words * 32), bool)
    bits[0, rng.integers(0, vocab, 9)] = True              # a few tokens
    bits[2] = True                                         # all but two
    bits[2, [3, 20]] = False
    r["allowed"] = np.packbits(bits, axis=1, bitorder="little").view(np.int32)      # mask 1 leaves nothing
    r["row_mask"] = np.array([0, 1, 2, -1, 2, 2, -1, 0, 1, -1, 2, -1, 0, 2])
    r["row_req"] = np.array([0, 0, 1, -1, 1, 2, 2, 3, -1, 3, 3, 4, 4, -1])
    z = (3 * rng.normal(size=(rows, vocab))).astype(np.float32)
    z[1], z[8] = np.nan, np.inf                            # nothing is left of these anyway
    z[2, 3], z[2, 20] = np.nan, np.inf                     # masked places
    z[3] = -np.inf
    z[4, 3] = np.inf
    z[4, 5] = np.nan                                       # left: conf is NaN
    z[5, [4, 7, 8]] = np.inf                               # they share the row
    r["ctx"][r["ctx"] == 4] = 0
    z[6] = 0.0
    z[9] = 2.5                                             # every token ties
    z[10] = torch.finfo(dtype).min
    z[11, : vocab - 1] = -np.inf
    z[11, vocab - 2] = -7.0
    z[13] = np.linspace(-3, 3, vocab)
    with np.errstate(all="ignore"):
        check_rules(B, z, r, vocab, reqs, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,pad,out_pad", [(7, 0, 2), (1000, 0, 5), (1000, 1, 0), (2003, 5, 2), (40001, 2, 3), (40001, 7, 15)])
def test_outputs_at_other_alignments_than_the_logits(B, dtype, vocab, pad, out_pad):
    """Rows of logits and of outputs start at different places within 16 bytes; what is stored is exact."""
    rng = np.random.default_rng(vocab + pad)
    rows, reqs = 21, 4
    r = make_rules(rng, rows, vocab, reqs, min(300, vocab), 10, 5)
    z = torch.from_numpy((3 * rng.normal(size=(rows, vocab))).astype(np.float32)).to(dtype)
    y = D.rules(z.float().numpy(), r["row_req"], vocab, **{k: v for k, v in r.items() if k != "row_req"})
    store = torch.full((rows, vocab + pad), 2.5, dtype=dtype, device="cuda")
    store[:, :vocab] = z.cuda()
    out = torch.full((rows, vocab + out_pad), 1.5, dtype=dtype, device="cuda")
    B.op_logit_rules(store[:, :vocab], to_rules(B, r, vocab, reqs), out=out[:, :vocab])
    assert torch.equal(out[:, :vocab].cpu(), torch.from_numpy(y).to(dtype))
    assert (out[:, vocab:] == 1.5).all()


@pytest.mark.parametrize("drop", ["ctx", "bias", "allowed", "row_req", "row_mask", "repetition", "presence", "frequency", "mask_id", "all"])
def test_rules_that_are_absent(B, drop):
    rng = np.random.default_rng(3)
    vocab, rows, reqs = 2003, 6, 6
    r = make_rules(rng, rows, vocab, reqs, 60, 6, 6)
    r["row_req"] = np.arange(6)
    r["row_mask"] = np.arange(6)
    z = (3 * rng.normal(size=(rows, vocab))).astype(np.float32)
    full = dict(r)
    gone = {"ctx": ["ctx", "begin", "gen", "end", "repetition", "presence", "frequency"], "bias": ["bias_at", "bias_tok", "bias_val"],
            "allowed": ["allowed", "row_mask"]}
    gone["all"] = gone["ctx"] + gone["bias"] + gone["allowed"]
    for k in gone.get(drop, [drop] if drop not in ("row_req", "row_mask") else []):
        full.pop(k)
    y = D.rules(z, r["row_req"], vocab, **{k: v for k, v in full.items() if k != "row_req"})
    if drop in ("row_req", "row_mask"):
        full.pop(drop)                                     # the binding's own default is the identity
    tok, conf = B.op_rules_confidence(f32(z), to_rules(B, full, vocab, reqs))
    t, c = D.confidence(y)
    assert np.array_equal(tok.cpu().numpy(), t) and (np.abs(host(conf) - c) <= c * CONF_TOL).all()
    assert np.array_equal(B.op_logit_rules(f32(z), to_rules(B, full, vocab, reqs)).cpu().numpy(), y)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,length", [(9000, 30000), (40001, 60000), (152064, 150000)])
def test_contexts_of_more_tokens_than_a_list_holds(B, dtype, vocab, length):
    """Thousands of different tokens in every share of the vocabulary: the touched entries are listed in turns."""
    rng = np.random.default_rng(length)
    r = make_rules(rng, 5, vocab, 2, 10, 300, 2)
    n = np.array([length, 7])
    end = np.cumsum(n)
    r.update(row_req=np.array([0, 0, 1, 0, -1]), ctx=rng.integers(0, vocab, int(end[-1])), begin=end - n, gen=end - n // 2, end=end)
    check_rules(B, (3 * rng.normal(size=(5, vocab))).astype(np.float32), r, vocab, 2, dtype)


def test_a_request_of_every_length_and_shared_tokens(B):
    """Contexts of no and one token, all of one token, contexts that overlap, and more biases than 16 bits number."""
    rng = np.random.default_rng(1)
    vocab, reqs = 70000, 6
    ctx = np.concatenate([np.full(5000, 17), rng.integers(0, vocab, 3000)])
    r = dict(row_req=np.arange(6), mask_id=5, ctx=ctx, begin=np.array([0, 0, 0, 4000, 7999, 3]), gen=np.array([0, 0, 100, 5000, 7999, 8000]),
             end=np.array([0, 1, 5000, 8000, 8000, 8000]), repetition=np.linspace(0.5, 2, 6).astype(np.float32),
             presence=np.linspace(-1, 1, 6).astype(np.float32), frequency=np.linspace(1, -1, 6).astype(np.float32))
    tok = np.sort(np.concatenate([rng.permutation(vocab)[:69000], [9, 9, 9, 69990, 69990]]))
    r.update(bias_at=np.array([0, 0, 0, 0, 3, 3, 3 + len(tok)]), bias_tok=np.concatenate([[17, 17, 18], tok]),
             bias_val=rng.normal(size=3 + len(tok)).astype(np.float32))
    check_rules(B, (3 * rng.normal(size=(6, vocab))).astype(np.float32), r, vocab, reqs, torch.float32)


@pytest.mark.parametrize("vocab,rows,reqs", [(33, 30000, 900), (1000, 9000, 9000), (40001, 1500, 30)])
def test_many_rows(B, vocab, rows, reqs):
    """Spans of more rows than are joined at once."""
    rng = np.random.default_rng(rows)
    r = make_rules(rng, rows, vocab, reqs, 12, 2, 16, density=0.4)
    z = (3 * rng.normal(size=(rows, vocab))).astype(np.float32)
    tok, conf = B.op_rules_confidence(f32(z), to_rules(B, r, vocab, reqs))
    out = B.op_logit_rules(f32(z), to_rules(B, r, vocab, reqs)).cpu().numpy()
    some = np.unique(np.concatenate([rng.integers(0, rows, 400), [0, rows - 1]]))
    part = {k: v for k, v in r.items() if k not in ("row_req", "row_mask")}
    y = D.rules(z[some], r["row_req"][some], vocab, row_mask=r["row_mask"][some], **part)
    t, c = D.confidence(y)
    assert np.array_equal(tok.cpu().numpy()[some], t) and (np.abs(host(conf)[some] - c) <= c * CONF_TOL).all()
    assert np.array_equal(out[some], y)


def test_rows_beyond_4_gib(B):
    """2^31 logits and more: the last rows are those of a small call, bit for bit."""
    vocab, rows = 152064, 14500
    z = torch.empty(rows, vocab, dtype=torch.bfloat16, device="cuda")
    z[:8].normal_()
    z[-8:].normal_()
    z[8:-8] = 1.0
    ctx = torch.randint(0, vocab, (500,), dtype=torch.int32, device="cuda")
    row_req = torch.zeros(rows, dtype=torch.int32, device="cuda")
    bounds = dict(ctx=ctx, ctx_begin=ints([0]), ctx_gen=ints([100]), ctx_end=ints([500]), repetition=f32([1.3]), presence=f32([0.2]))
    rules = B.logit_rules(vocab, row_req, 1, mask_id=vocab - 1, **bounds)
    tok, conf = B.op_rules_confidence(z, rules)
    t, c = B.op_rules_confidence(z[-8:].clone(), rules)
    assert torch.equal(tok[-8:], t) and torch.equal(conf[-8:], c)
    want = B.op_logit_rules(z[-8:].clone(), rules)
    B.op_logit_rules(z, rules)
    assert torch.equal(z[-8:], want) and bool(torch.isinf(z[:, -1]).all())


# ---- indices that are out of range ----------------------------------------------------------------------------

def test_bad_indices_are_skipped_and_flagged(B):
    rng = np.random.default_rng(8)
    vocab, rows, reqs = 1500, 8, 4
    r = make_rules(rng, rows, vocab, reqs, 40, 0, 3, density=0.5)
    r["row_req"], r["row_mask"] = np.array([0, 1, 1, 2, 3, 0, 2, 3]), np.array([0, 1, 2, -1, 0, 1, 2, -1])
    z = (3 * rng.normal(size=(rows, vocab))).astype(np.float32)
    y = D.rules(z, r["row_req"], vocab, **{k: v for k, v in r.items() if k != "row_req"})
    t, c = D.confidence(y)

    def run(change, skipped=()):
        bad = {k: np.array(v) if not np.isscalar(v) else v for k, v in r.items()}
        change(bad)
        rules, flag = to_rules(B, bad, vocab, reqs), new_flag()
        tok, conf = B.op_rules_confidence(f32(z), rules, error_flag=flag)
        assert int(flag) >= 100
        flag.zero_()
        out = torch.full((rows, vocab), 7.0, device="cuda")
        B.op_logit_rules(f32(z), rules, out=out, error_flag=flag)
        assert int(flag) >= 100
        B.op_rules_confidence(f32(z), rules)               # nobody asks
        good = np.setdiff1d(np.arange(rows), skipped)
        return tok.cpu().numpy(), host(conf), out.cpu().numpy(), good

    for name, value in (("row_req", reqs), ("row_req", -2), ("row_req", 1 << 30), ("row_mask", 3), ("row_mask", -2)):
        def change(b, name=name, value=value):
            b[name][[2, 7]] = value
        tok, conf, out, good = run(change, [2, 7])
        assert np.array_equal(tok[good], t[good]) and (np.abs(conf - c)[good] <= c[good] * CONF_TOL).all()
        assert np.array_equal(out[good], y[good]) and (tok[[2, 7]] == -1).all() and (conf[[2, 7]] == 0).all() and (out[[2, 7]] == 7).all()

    def ids(b):                                            # ids that are no tokens: as if they were not there
        at = b["end"][1] - 1
        b["ctx"][at] = vocab + 5
        b["ctx"][b["begin"][3]] = -1
    tok, _, out, good = run(ids, [1, 2, 4, 7])
    assert np.array_equal(tok[good], t[good]) and np.array_equal(out[good], y[good])

    for k, value in (("begin", -1), ("end", len(r["ctx"]) + 1), ("gen", -3), ("end", -1), ("gen", 1 << 30)):
        def bounds(b, k=k, value=value):                   # request 1 then has no context
            b[k][1] = value
        _, _, out, good = run(bounds, [1, 2])
        assert np.array_equal(out[good], y[good])
        empty = dict(r, begin=np.where(np.arange(4) == 1, 0, r["begin"]), gen=np.where(np.arange(4) == 1, 0, r["gen"]),
                     end=np.where(np.arange(4) == 1, 0, r["end"]))
        assert np.array_equal(out[[1, 2]], D.rules(z, r["row_req"], vocab, **{k2: v for k2, v in empty.items() if k2 != "row_req"})[[1, 2]])


def test_biases_out_of_order_or_range_raise_the_flag(B):
    vocab = 500
    z = torch.randn(2, vocab, device="cuda")
    for tok in ([5, 4], [5, 500], [-1, 3], [2, 1 << 30]):
        flag = new_flag()
        rules = B.logit_rules(vocab, None, 2, bias_at=ints([0, 0, 2]), bias_tok=ints(tok), bias_val=f32([1, 1]))
        out = B.op_logit_rules(z, rules, out=torch.empty_like(z), error_flag=flag)
        assert int(flag) >= 100 and torch.equal(out[0], z[0])
    for at in ([0, 3, 2], [0, 0, 3], [0, -1, 2]):
        flag = new_flag()
        rules = B.logit_rules(vocab, None, 2, bias_at=ints(at), bias_tok=ints([1, 2]), bias_val=f32([1, 1]))
        B.op_rules_confidence(z, rules, error_flag=flag)
        assert int(flag) >= 100


# ---- streams, graphs, calls at once ---------------------------------------------------------------------------

def test_captured_calls_read_what_the_tensors_hold_then(B):
    rng = np.random.default_rng(2)
    vocab, rows, reqs = 40001, 12, 3
    first, second = (make_rules(np.random.default_rng(s), rows, vocab, reqs, 50, 0, 4) for s in (1, 2))
    n = max(len(first["ctx"]), len(second["ctx"]))
    for r in (first, second):
        r["ctx"] = np.concatenate([r["ctx"], np.zeros(n - len(r["ctx"]), np.int64)])
        r["bias_at"], r["bias_tok"], r["bias_val"] = np.array([0, 1, 2, 3]), np.array([3, 4, 5]), np.ones(3, np.float32)
    z = [(3 * rng.normal(size=(rows, vocab))).astype(np.float32) for _ in range(2)]
    live, buf = to_rules(B, first, vocab, reqs), f32(z[0])
    x = torch.randn(40, 200, device="cuda")
    w, sw = B.op_quant_i8(torch.randn(300, 200, device="cuda"))
    B.op_rules_confidence(buf, live)
    B.op_gemm_i8(*B.op_quant_i8(x), w, sw)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tok, conf = B.op_rules_confidence(buf, live)
        out = B.op_logit_rules(buf, live, out=torch.empty_like(buf))
        y = B.op_gemm_i8(*B.op_quant_i8(x), w, sw)
    for r, zz in ((first, z[0]), (second, z[1])):
        fresh = to_rules(B, r, vocab, reqs)
        for a, b in zip(live.tensors, fresh.tensors):
            a.copy_(b)
        buf.copy_(f32(zz))
        x.normal_()
        g.replay()
        torch.cuda.synchronize()
        t, c = B.op_rules_confidence(buf, fresh)
        assert torch.equal(tok, t) and torch.equal(conf, c)
        assert torch.equal(out, B.op_logit_rules(buf, fresh, out=torch.empty_like(buf)))
        assert torch.equal(y, B.op_gemm_i8(*B.op_quant_i8(x), w, sw))
        assert np.array_equal(out.cpu().numpy(), D.rules(zz, r["row_req"], vocab, **{k: v for k, v in r.items() if k != "row_req"}))


FIRST_CALL = """
import torch
from paper_2607_08930_b200 import binding as B
torch.manual_seed(0)
x, w = torch.randn(200, 700, device="cuda"), torch.randn(900, 700, device="cuda")
ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
rules = B.logit_rules(900, None, 200, mask_id=7, ctx=ints(3, 4, 4, 9), ctx_begin=torch.zeros(200, dtype=torch.int32, device="cuda"),
                      ctx_gen=torch.ones(200, dtype=torch.int32, device="cuda"),
                      ctx_end=torch.full((200,), 4, dtype=torch.int32, device="cuda"), frequency=torch.ones(200, device="cuda"))
def step():
    wq, sw = B.op_quant_i8(w)
    y = B.op_gemm_i8(*B.op_quant_i8(x), wq, sw, mode=2)
    return (y, *B.op_rules_confidence(y, rules), B.op_logit_rules(y, rules, out=torch.empty_like(y)))
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    got = step()
g.replay()
torch.cuda.synchronize()
want = step()
assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.isfinite(got[0]).all()
print("same")
"""


def test_the_first_call_of_a_process_may_be_captured(B):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALL], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]


def test_calls_on_two_streams_at_once(B):
    """No workspace is shared: calls side by side give what they give alone, and the same every time."""
    rng = np.random.default_rng(4)
    jobs = []
    for s in range(2):
        r = make_rules(rng, 40, 30011, 5, 200, 9, 40)
        z = f32((3 * rng.normal(size=(40, 30011))).astype(np.float32))
        x, w = torch.randn(150, 1000, device="cuda").bfloat16(), torch.randn(520, 1000, device="cuda")
        rules, wq = to_rules(B, r, 30011, 5), B.op_quant_i8(w)

        def job(z=z, rules=rules, x=x, wq=wq):
            t, c = B.op_rules_confidence(z, rules)
            return t, c, B.op_logit_rules(z, rules, out=torch.empty_like(z)), B.op_gemm_i8(*B.op_quant_i8(x), *wq, mode=2)
        jobs.append(job)
    alone = [job() for job in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(10):
        got = []
        for job, s in zip(jobs, streams):
            with torch.cuda.stream(s):
                got.append(job())
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_the_kernel_before_is_waited_for(B):
    """Codes made, multiplied and reduced in one go, many times: each call reads what the one before it wrote."""
    x = torch.randn(64, 512, device="cuda").bfloat16()
    w = torch.randn(700, 512, device="cuda")
    want = None
    for _ in range(50):
        wq, sw = B.op_quant_i8(w)                          # the weights too are written right before the product
        y = B.op_gemm_i8(*B.op_quant_i8(x), wq, sw, mode=2)
        tok, conf = B.op_rules_confidence(y, B.logit_rules(700, None, 64))
        z = B.op_logit_rules(y, B.logit_rules(700, None, 64, mask_id=3))
        got = (y, tok, conf, z)
        want = want or got
        assert all(torch.equal(a, b) for a, b in zip(want, got))


# ---- projections ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("mode", [0, 1, 2])
@pytest.mark.parametrize("m,n,k", [(1, 130, 20000), (16, 640, 9000), (33, 300, 4000), (64, 128, 131071), (128, 520, 6000),
                                   (200, 384, 18944), (256, 1000, 5000), (512, 3584, 2000)])
def test_long_sums_shared_by_clusters(B, m, n, k, mode):
    check_gemm(B, m, n, k, mode)


@pytest.mark.parametrize("mode", [0, 2, 3])
def test_many_items_a_cta(B, mode):
    check_gemm(B, 3000, 2500, 300, mode)
    check_gemm(B, 90, 30000, 200, mode)


def test_rows_of_codes_and_outputs_beyond_4_gib(B):
    """Row strides of 2^20: the last rows are those of a dense call, bit for bit."""
    a = torch.empty(4200, 1 << 20, dtype=torch.int8, device="cuda")[:, :300]
    a.random_(-128, 128)
    w, sw = B.op_quant_i8(torch.randn(140, 300, device="cuda"))
    sa = torch.rand(4200, device="cuda")
    out = torch.empty(4200, 1 << 20, dtype=torch.bfloat16, device="cuda")[:, :140]
    B.op_gemm_i8(a, sa, w, sw, C_out=out)
    dense = B.i8_codes(4200, 300)
    dense.copy_(a)
    assert torch.equal(out, B.op_gemm_i8(dense, sa, w, sw))
    del a, dense
    x = torch.randn(16, 140, device="cuda").bfloat16()
    out[-16:] = x
    far, s = B.op_quant_i8(out)
    near, s2 = B.op_quant_i8(x)
    assert torch.equal(far[-16:], near) and torch.equal(s[-16:], s2)


def test_outputs_on_inputs_are_refused(B):
    buf = torch.zeros(1 << 16, dtype=torch.int8, device="cuda")
    a = buf[:4096].view(16, 256)
    w, sw = B.op_quant_i8(torch.randn(64, 256, device="cuda"))
    with pytest.raises(B.BlockServeError):
        B.op_gemm_i8(a, torch.ones(16, device="cuda"), w, sw, C_out=buf[:2048].view(torch.bfloat16).view(16, 64))
    x = torch.zeros(16, 256, device="cuda")
    with pytest.raises(B.BlockServeError):
        B.op_quant_i8(x, codes=x.view(torch.int8)[:, :256])
    z = torch.zeros(4, 64, device="cuda")
    with pytest.raises(B.BlockServeError):
        B.op_logit_rules(z[:3], B.logit_rules(64, None, 3), out=z[1:])


@pytest.fixture()
def debug_lib(B, monkeypatch):
    from paper_2607_08930_b200 import build
    path = build.build(debug=True)
    regular = B.lib()
    monkeypatch.setattr(B, "LIB_PATH", path)
    monkeypatch.setattr(B, "_lib", None)
    assert B.lib() is not regular
    return B


@pytest.mark.parametrize("mode", [0, 1, 2, 3])
@pytest.mark.parametrize("m,n,k,after", [(20, 130, 400, 0), (20, 130, 400, 3), (16, 640, 9000, 40), (300, 384, 9000, 7),
                                         (700, 5000, 700, 2), (3000, 2500, 300, 1)])
def test_a_wait_that_runs_out_leaves_no_result(debug_lib, m, n, k, after, mode):
    """In the bounds-checked build the wait for k step b runs out when the flag holds -1 - b (the first CTA that gives up
    raises it, so later ones may go on): outputs are NaN or right, the flag says so, and the next call is right."""
    B = debug_lib
    rng = np.random.default_rng(m + after)
    _, ta = random_codes(rng, m, k)
    _, tw = random_codes(rng, n, k)
    _, tw2 = random_codes(rng, n, k)
    sa, sw = f32(rng.random(m)), f32(rng.random(n) / k)
    flag = torch.full((1,), -1 - after, dtype=torch.int32, device="cuda")

    def run():
        out = torch.zeros(m, n, dtype=torch.float32 if mode in (1, 2) else torch.bfloat16, device="cuda")
        return host(B.op_gemm_i8(ta, sa, tw, sw, mode=mode, W2=tw2 if mode == 3 else None, w2_scale=sw if mode == 3 else None,
                                 C_out=out, error_flag=flag))
    got = run()
    assert int(flag) == 1
    flag.zero_()
    want = run()
    assert int(flag) == 0 and np.isfinite(want).all()
    lost = np.isnan(got)
    assert lost.any() and np.array_equal(got[~lost], want[~lost])


# ---- the operators together -----------------------------------------------------------------------------------

@pytest.mark.parametrize("m,d,ffn", [(1, 256, 704), (40, 256, 704), (300, 384, 1000), (64, 3584, 1200)])
def test_a_feed_forward_block(B, m, d, ffn):
    """x + down(silu(gate(norm x)) up(norm x)) through codes, against the same in 64 bits on the codes of each stage: the
    bounds are those of the stages, and of their codes the last halves."""
    rng = np.random.default_rng(m + d)
    x = torch.from_numpy(rng.normal(size=(m, d)).astype(np.float32)).cuda()
    gain = torch.from_numpy(1 + 0.1 * rng.normal(size=d)).bfloat16().cuda()
    gate, up, down = (B.op_quant_i8(f32(rng.normal(size=s) / np.sqrt(s[1])))
                      for s in ((ffn, d), (ffn, d), (d, ffn)))
    a, sa = B.op_quant_i8(x, gain=gain, eps=1e-6)
    h = B.op_gemm_i8(a, sa, *gate, mode=3, W2=up[0], w2_scale=up[1])
    b, sb = B.op_quant_i8(h)
    out = x.clone()
    B.op_gemm_i8(b, sb, *down, mode=1, C_out=out)
    y, _, _ = D.quant(host(x), host(gain), 1e-6)
    assert (np.abs(host(a) * host(sa)[:, None] - y) <= host(sa)[:, None] * 0.51).all()
    z, u = D.gemm(host(a), host(sa), host(gate[0]), host(gate[1])), D.gemm(host(a), host(sa), host(up[0]), host(up[1]))
    ref = z / (1 + np.exp(-z)) * u
    assert (np.abs(host(h) - ref) <= np.abs(ref) * (HALF_BF16 + (20 + 6 * np.abs(z)) * HALF_F32) + 1e-37).all()
    _, codes, scale = D.quant(host(h))
    assert np.array_equal(host(b), codes) and np.array_equal(host(sb), scale)
    ref = D.gemm(codes, scale, host(down[0]), host(down[1]))
    assert (np.abs(host(out) - (host(x) + ref)) <= np.abs(host(x) + ref) * HALF_F32 + np.abs(ref) * 3.1 * HALF_F32 + 1e-38).all()


@pytest.mark.parametrize("reqs,block,vocab,d", [(1, 1, 1024, 256), (3, 32, 1024, 256), (4, 32, 2000, 384), (16, 32, 152064, 256)])
def test_a_constrained_block_step(B, reqs, block, vocab, d):
    """Hidden states -> codes -> LM head -> rules -> token and confidence, as a denoising step under a grammar runs them; the
    logits after the rules give the same tokens through op_confidence."""
    rng = np.random.default_rng(vocab + reqs)
    rows = reqs * block
    x = torch.from_numpy(rng.normal(size=(rows + 5, d)).astype(np.float32)).cuda()
    idx = rng.permutation(rows + 5)[:rows]
    gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    head = B.op_quant_i8(torch.randn(vocab, d, device="cuda") * 0.2)
    codes, scale = B.op_quant_i8(x, gain=gain, idx=ints(idx))
    logits = B.op_gemm_i8(codes, scale, *head, mode=2)
    r = make_rules(rng, rows, vocab, reqs, 200, 20, rows)
    r["row_req"] = np.repeat(np.arange(reqs), block)
    r["row_mask"] = np.where(np.arange(rows) % 3 == 0, -1, np.arange(rows))
    rules = to_rules(B, r, vocab, reqs)
    flag = new_flag()
    tok, conf = B.op_rules_confidence(logits, rules, error_flag=flag)
    y = D.rules(logits.cpu().numpy(), r["row_req"], vocab, **{k: v for k, v in r.items() if k != "row_req"})
    t, c = D.confidence(y)
    assert np.array_equal(tok.cpu().numpy(), t) and (np.abs(host(conf) - c) <= c * CONF_TOL).all()
    ruled = B.op_logit_rules(logits, rules, error_flag=flag)
    assert np.array_equal(ruled.cpu().numpy(), y) and int(flag) == 0
    left = t >= 0
    tok2, conf2 = B.op_confidence(ruled, vocab - 1)
    assert np.array_equal(tok2.cpu().numpy()[left], t[left])
    assert (np.abs(host(conf2) - c)[left] <= c[left] * 2.0 ** -15).all()
