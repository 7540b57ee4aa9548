"""8-bit row codes, 8-bit projections, rules on logits and the confidence under them, against the 64-bit oracle (needs a
B200)."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as D

pytestmark = pytest.mark.gpu

HALF_BF16, HALF_F32 = 2.0 ** -8, 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    from paper_2607_08930_b200 import build
    build.build()
    from paper_2607_08930_b200 import binding
    return binding


def host(t):
    return t.detach().cpu().double().numpy()


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def f32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()


# ---- 8-bit row codes -----------------------------------------------------------------------------------------

def strided(x, pad, offset=0):
    """The same rows `pad` elements further apart, starting `offset` elements into their storage, among NaN."""
    m, k = x.shape
    store = torch.full((m * (k + pad) + offset + 64,), float("nan"), dtype=x.dtype, device="cuda")
    view = store[offset:offset + m * (k + pad)].view(m, k + pad)[:, :k]
    view.copy_(x)
    return view


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,k,pad,offset", [(1, 1, 0, 0), (3, 7, 0, 0), (5, 33, 0, 0), (4, 256, 8, 0), (17, 384, 0, 0),
                                            (9, 1000, 1, 0), (2, 1001, 0, 3), (64, 3584, 0, 0), (33, 4096, 16, 8),
                                            (3, 18944, 0, 0), (2, 32768, 0, 0), (2, 32769, 0, 1), (2, 100003, 5, 0)])
def test_codes_are_the_exact_quotients_rounded(B, dtype, m, k, pad, offset):
    rng = np.random.default_rng(m * k)
    x = rng.normal(size=(m, k)) * 2.0 ** rng.integers(-20, 20, (m, 1))
    x = torch.from_numpy(x).to(dtype)
    x[0, : k // 2] = x[0].abs().max() * torch.linspace(-1, 1, k // 2 if k > 1 else 0).to(dtype)     # many near-halves
    y, codes, scale = D.quant(host(x))
    got, s = B.op_quant_i8(strided(x.cuda(), pad, offset))
    assert np.array_equal(host(s), scale)
    assert np.array_equal(host(got), codes)


def test_quotients_at_and_next_to_halves(B):
    """Rows of one largest element (127 times an odd scale, whose scale fp32 holds) and elements within two steps of every
    half multiple of that scale."""
    rng = np.random.default_rng(5)
    rows = []
    for _ in range(64):
        s = np.float32(rng.uniform(1, 2)) * np.float32(2.0) ** rng.integers(-100, 100)
        top = np.float32(127 * np.float64(s))
        s = top * np.float32(1 / 127)
        half = ((np.arange(-127, 127) + 0.5) * np.float64(s)).astype(np.float32)
        near = [half]
        for _ in range(2):
            near += [np.nextafter(near[-1], np.float32(np.inf)), ]
        low = half
        for _ in range(2):
            low = np.nextafter(low, np.float32(-np.inf))
            near.append(low)
        row = np.concatenate(near)
        rows.append(np.concatenate([row[np.abs(row) <= top], np.full(2000, top)])[:2000])
    x = np.stack([r[:1200] for r in rows])
    x[:, 0] = [r[-1] for r in rows]
    _, codes, scale = D.quant(x)
    got, s = B.op_quant_i8(f32(x))
    assert np.array_equal(host(s), scale) and np.array_equal(host(got), codes)


def test_scales_at_the_ends_of_the_range(B):
    """Zeros, subnormals, the largest values, and rows with infinities or NaN among others."""
    x = np.zeros((9, 300), np.float32)
    x[1, 5] = 2.0 ** -149
    x[2] = np.linspace(-1, 1, 300).astype(np.float32) * np.float32(2.0 ** -127)
    x[3] = np.linspace(-1, 1, 300).astype(np.float32) * np.finfo(np.float32).max
    x[4] = np.linspace(-1, 1, 300)
    x[5, 7] = np.inf
    x[6, 299] = np.nan
    x[7] = np.linspace(-1, 1, 300).astype(np.float32) * np.float32(127 * 2.0 ** -126)
    x[8, 0] = -np.inf
    _, codes, scale = D.quant(x)
    got, s = B.op_quant_i8(f32(x))
    assert np.array_equal(host(s), scale, equal_nan=True) and np.array_equal(host(got), codes)
    assert np.isnan(host(s)[[5, 6, 8]]).all() and (host(s)[:3] == 2.0 ** -126).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,k", [(1, 9), (33, 384), (7, 3584), (4, 18944), (2, 40001)])
def test_codes_of_rms_norms(B, dtype, m, k):
    """y in fp32: a sum of squares of at most 32 terms a thread (long rows: k / 1024) and ten joins, its root and two
    products: relative error below delta.  A code is then within 127 * 2 delta of a rounded quotient."""
    rng = np.random.default_rng(k)
    x = torch.from_numpy(rng.normal(size=(m + 5, k)) * 2.0 ** rng.integers(-3, 4, (m + 5, 1))).to(dtype)
    gain = torch.from_numpy(1 + 0.2 * rng.normal(size=k)).bfloat16()
    idx = rng.permutation(m + 5)[:m]
    y, _, scale = D.quant(host(x)[idx], host(gain), 1e-5)
    got, s = B.op_quant_i8(x.cuda(), gain=gain.cuda(), eps=1e-5, idx=ints(idx))
    delta = (max(32, k / 1024) + 10 + 8) * HALF_F32
    assert (np.abs(host(s) - scale) <= scale * (delta + 2 * HALF_F32)).all()
    assert (np.abs(host(got) - y / host(s)[:, None]) <= 0.5 + 127 * 2 * delta).all()


def test_gathered_rows_out_of_range_are_skipped_and_flagged(B):
    x = torch.randn(6, 200).cuda()
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    codes, scale = B.i8_codes(5, 200), torch.full((5,), -7.0, device="cuda")
    codes.fill_(99)
    B.op_quant_i8(x, idx=ints([2, 6, 0, -1, 5]), codes=codes, scale=scale, error_flag=flag)
    assert int(flag) >= 100
    ref, s = B.op_quant_i8(x, idx=ints([2, 0, 5]))
    assert torch.equal(codes[[0, 2, 4]], ref) and torch.equal(scale[[0, 2, 4]], s)
    assert (codes[[1, 3]] == 99).all() and (scale[[1, 3]] == -7).all()


def test_bytes_behind_a_row_of_codes_are_left(B):
    x = torch.randn(7, 37).cuda()
    store = torch.full((7, 64), 55, dtype=torch.int8, device="cuda")
    B.op_quant_i8(x, codes=store[:, :37])
    assert (store[:, 37:] == 55).all()


# ---- 8-bit projections ---------------------------------------------------------------------------------------

def random_codes(rng, rows, k, pad=0):
    c = rng.integers(-128, 128, (rows, k)).astype(np.int8)
    ld = (k + 15) // 16 * 16 + pad
    store = np.full((rows, ld), 77, np.int8)               # what lies between the rows must not matter
    store[:, :k] = c
    return c, torch.from_numpy(store).cuda()[:, :k]


def check_gemm(B, m, n, k, mode, pad=0, cpad=0, seed=0):
    rng = np.random.default_rng(seed + m + 3 * n + 7 * k + mode)
    a, ta = random_codes(rng, m, k, pad)
    w, tw = random_codes(rng, n, k, pad)
    sa = (2.0 ** rng.uniform(-8, -2, m)).astype(np.float32)
    sw = (2.0 ** rng.uniform(-14, -10, n) / np.sqrt(k)).astype(np.float32)
    z = D.gemm(a, sa, w, sw)
    dtype = torch.float32 if mode in (1, 2) else torch.bfloat16
    store = torch.full((m, n + cpad), 3.0, dtype=dtype, device="cuda")
    out = store[:, :n]
    err = np.abs(z) * 3 * HALF_F32                         # sum to fp32, two products
    if mode == 3:
        w2, tw2 = random_codes(rng, n, k, pad)
        sw2 = (2.0 ** rng.uniform(-14, -10, n) / np.sqrt(k)).astype(np.float32)
        u = D.gemm(a, sa, w2, sw2)
        got = B.op_gemm_i8(ta, f32(sa), tw, f32(sw), mode=3, W2=tw2, w2_scale=f32(sw2), C_out=out)
        ref = z / (1 + np.exp(-z)) * u
        # the exponent's argument is off by 4 half steps, 2^x and 1/x by 2^-22, the products by a half step each
        tol = np.abs(ref) * (HALF_BF16 + (20 + 6 * np.abs(z)) * HALF_F32) + 1e-37
    else:
        base = None
        if mode == 1:
            base = rng.normal(size=(m, n)).astype(np.float32)
            out.copy_(f32(base))
        got = B.op_gemm_i8(ta, f32(sa), tw, f32(sw), mode=mode, C_out=out)
        ref = z if base is None else base + z
        tol = err * 1.01 + np.abs(ref) * (HALF_BF16 if mode == 0 else HALF_F32 if mode == 1 else 0) + 1e-38
    assert got.data_ptr() == out.data_ptr()
    off = np.abs(host(out) - ref) - tol
    assert (off <= 0).all(), (float(off.max()), np.argwhere(off > 0)[:4])
    if cpad:
        assert (store[:, n:] == 3.0).all()
    return out


@pytest.mark.parametrize("mode", [0, 1, 2, 3])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 24, 16), (3, 130, 33), (16, 128, 128), (17, 257, 129), (31, 1000, 384),
                                   (64, 704, 256), (64, 384, 1000), (100, 2000, 384), (128, 640, 2100), (129, 384, 256),
                                   (200, 1000, 384), (256, 4608, 3584), (257, 520, 300), (512, 704, 256), (700, 2000, 130),
                                   (1025, 1300, 513)])
def test_products(B, m, n, k, mode):
    check_gemm(B, m, n, k, mode)


@pytest.mark.parametrize("mode", [0, 1, 2, 3])
@pytest.mark.parametrize("m,n,k,pad,cpad", [(5, 130, 200, 16, 6), (70, 264, 384, 48, 8), (300, 520, 777, 16, 3), (300, 520, 777, 0, 24)])
def test_products_of_strided_rows(B, m, n, k, pad, cpad, mode):
    check_gemm(B, m, n, k, mode, pad, cpad)


def test_the_largest_sums(B):
    """Codes of -128 throughout, at the longest K: the sum is just below 2^31."""
    k = B.I8_MAX_K
    for m in (1, 130):
        a = torch.full((m, k + 1), -128, dtype=torch.int8, device="cuda")[:, :k]
        w = torch.full((3, k + 1), -128, dtype=torch.int8, device="cuda")[:, :k]
        w[1] = 127
        one = torch.ones(256, device="cuda")
        got = host(B.op_gemm_i8(a, one[:m], w, one[:3], mode=2))
        ref = np.array([16384.0, -16256.0, 16384.0]) * k
        assert (np.abs(got - ref) <= np.abs(ref) * HALF_F32).all()


def test_rows_without_a_scale_are_nan(B):
    rng = np.random.default_rng(3)
    a, ta = random_codes(rng, 40, 256)
    w, tw = random_codes(rng, 300, 256)
    sa, sw = np.ones(40, np.float32), np.ones(300, np.float32)
    sa[7], sw[11] = np.nan, np.nan
    got = host(B.op_gemm_i8(ta, f32(sa), tw, f32(sw)))
    bad = np.isnan(got)
    assert bad[7].all() and bad[:, 11].all() and bad.sum() == 300 + 39


# ---- rules on logits -----------------------------------------------------------------------------------------

def make_rules(rng, rows, vocab, reqs, ctx_len=40, biases=5, masks=0, mask_id=None, density=None, dups=True):
    """Rules of `reqs` requests as numpy arrays: contexts with repeated and masked tokens, biases with equal neighbours."""
    mask_id = vocab - 1 if mask_id is None else mask_id
    row_req = np.sort(rng.integers(0, reqs, rows))
    n = rng.integers(0, ctx_len + 1, reqs)
    end = np.cumsum(n)
    ctx = np.minimum((vocab * rng.random(int(end[-1])) ** 2).astype(np.int64), vocab - 1)
    ctx[rng.random(len(ctx)) < 0.1] = max(mask_id, 0)
    b = rng.integers(0, biases + 1, reqs)
    tok = [np.sort(rng.integers(0, vocab, c) if dups else rng.choice(vocab, min(c, vocab), replace=False)) for c in b]
    b = [len(t) for t in tok]
    r = dict(row_req=row_req, mask_id=mask_id, ctx=ctx, begin=end - n, gen=end - n + (n * rng.random(reqs)).astype(int), end=end,
             repetition=rng.uniform(0.7, 1.6, reqs).astype(np.float32), presence=rng.uniform(-0.5, 0.8, reqs).astype(np.float32),
             frequency=rng.uniform(-0.2, 0.5, reqs).astype(np.float32), bias_at=np.concatenate([[0], np.cumsum(b)]),
             bias_tok=np.concatenate(tok + [np.zeros(0, np.int64)]), bias_val=(3 * rng.normal(size=sum(b))).astype(np.float32))
    if masks:
        words = (vocab + 31) // 32
        d = rng.choice([0.0, 0.001, 0.3, 0.97], masks) if density is None else np.full(masks, density)
        bits = rng.random((masks, words * 32)) < d[:, None]
        r["allowed"] = np.packbits(bits, axis=1, bitorder="little").view(np.int32)
        r["row_mask"] = rng.integers(-1, masks, rows)
    return r


def to_rules(B, r, vocab, reqs):
    g = lambda k, f: None if r.get(k) is None else f(r[k])              # noqa: E731
    return B.logit_rules(vocab, g("row_req", ints), reqs, mask_id=r.get("mask_id", -1), ctx=g("ctx", ints),
                         ctx_begin=g("begin", ints), ctx_gen=g("gen", ints), ctx_end=g("end", ints),
                         repetition=g("repetition", f32), presence=g("presence", f32), frequency=g("frequency", f32),
                         bias_at=g("bias_at", ints), bias_tok=g("bias_tok", ints), bias_val=g("bias_val", f32),
                         allowed=g("allowed", ints), row_mask=g("row_mask", ints))


# conf = 1 / sum exp(z - max): a term is off by 2^-22 (2^x) and three half steps of z - max (its weight falls faster than
# that grows: at most log V of them on average), the sum by a half step for each of the up to 70 values that a thread, a
# warp and the join add one after the other
CONF_TOL = 2.0 ** -17


def check_rules(B, z, r, vocab, reqs, dtype):
    z = torch.from_numpy(z).to(dtype)
    rows = z.shape[0]
    y = D.rules(z.float().numpy(), r["row_req"], vocab, **{k: v for k, v in r.items() if k != "row_req"})
    rules = to_rules(B, r, vocab, reqs)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    want = torch.from_numpy(y).to(dtype)
    for pad in (0, 3, 16):                                  # rows at any alignment
        store = torch.full((rows, vocab + pad), 2.5, dtype=dtype, device="cuda")
        store[:, :vocab] = z.cuda()
        view = store[:, :vocab]
        tok, conf = B.op_rules_confidence(view, rules, error_flag=flag)
        t, c = D.confidence(y)
        assert np.array_equal(tok.cpu().numpy(), t), (pad, np.flatnonzero(tok.cpu().numpy() != t)[:5])
        got = host(conf)
        assert np.array_equal(np.isnan(got), np.isnan(c))
        assert (np.abs(got - c) <= c * CONF_TOL)[~np.isnan(c)].all()
        out = torch.full((rows, vocab + pad), 1.5, dtype=dtype, device="cuda")
        B.op_logit_rules(view, rules, out=out[:, :vocab], error_flag=flag)
        assert torch.equal(view.cpu().nan_to_num(7.0, 8.0, 9.0), z.nan_to_num(7.0, 8.0, 9.0))      # read only
        B.op_logit_rules(view, rules, error_flag=flag)      # in place
        for x in (out, store):
            assert torch.equal(x[:, :vocab].cpu().nan_to_num(123.0, 124.0, 125.0), want.nan_to_num(123.0, 124.0, 125.0)), pad
        assert (out[:, vocab:] == 1.5).all() and (store[:, vocab:] == 2.5).all()
    assert int(flag) == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,rows,reqs,ctx_len,biases,masks", [
    (1, 3, 2, 3, 1, 0), (2, 4, 3, 5, 2, 2), (31, 5, 5, 20, 4, 3), (32, 5, 2, 40, 8, 3), (33, 9, 4, 40, 8, 9), (1000, 12, 3, 300, 20, 12),
    (1024, 4, 4, 160, 8, 4), (2003, 70, 20, 500, 30, 40), (16385, 10, 4, 2000, 100, 5), (40001, 33, 9, 900, 50, 33),
    (126464, 40, 3, 4000, 300, 4), (152064, 7, 7, 3000, 100, 7), (200003, 3, 2, 20000, 10, 2)])
def test_rules_and_confidence(B, dtype, vocab, rows, reqs, ctx_len, biases, masks):
    rng = np.random.default_rng(vocab + rows)
    r = make_rules(rng, rows, vocab, reqs, ctx_len, biases, masks)
    check_rules(B, (rng.normal(size=(rows, vocab)) * 3).astype(np.float32), r, vocab, reqs, dtype)
