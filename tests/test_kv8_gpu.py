"""Per-head norms with rotation, the 8-bit KV cache and attention over it against the 64-bit oracle (needs a B200)."""
import numpy as np
import pytest
import torch

from oracle import blockserve_oracle as O
from oracle import kv8_oracle as K

pytestmark = pytest.mark.gpu
THETA, EPS = 10000.0, 1e-6
HALF_BF16 = torch.finfo(torch.bfloat16).eps / 2


@pytest.fixture(scope="module")
def B():
    from paper_2607_08930_b200 import build
    build.build()
    from paper_2607_08930_b200 import binding
    return binding


def bf16(a):
    return torch.from_numpy(np.asarray(a, np.float32)).to(torch.bfloat16)


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def host(t):
    return t.detach().double().cpu().numpy()


def slabs(rng, lengths, gap=True):
    """kv_base of slabs of whole blocks in shuffled order; the total number of blocks."""
    base, free = np.zeros(len(lengths), np.int64), 1
    for i in rng.permutation(len(lengths)):
        base[i] = free * 32
        free += (int(lengths[i]) + 31) // 32 + (int(rng.integers(0, 2)) if gap else 0)
    return base, free + 1


def prefix(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int64)


def random_cache(rng, blocks, hkv, dh, spread=4):
    """Codes over the whole range (no NaN) and power-of-two scales 2^-spread .. 2^spread."""
    codes = rng.integers(0, 127, (blocks, hkv, 32, dh)).astype(np.uint8) + 128 * rng.integers(0, 2, (blocks, hkv, 32, dh)).astype(np.uint8)
    return codes, 2.0 ** (rng.integers(-spread, spread + 1, (blocks, hkv)) - 7.0)


def to_gpu(codes, scales):
    return (torch.from_numpy(np.ascontiguousarray(codes)).cuda().view(torch.float8_e4m3fn),
            torch.from_numpy(np.ascontiguousarray(scales.astype(np.float32))).cuda())


# fp32 chain of the norm and the rotation: the mean of dh squares (sixteen serial sums per lane, then a tree: a relative
# error under 19 2^-24, half of it after the root - (dh / 8 + 8) 2^-24 and more is allowed), rsqrtf (2^-22), three products
# and a sum of two, the table's own 2^-24
def chain_tol(x, dh):
    half = dh // 2
    pair = np.abs(x[..., :half]) + np.abs(x[..., half:])
    return np.concatenate([pair, pair], -1) * (dh / 8 + 8 + 4 + 8) * 2.0 ** -24


NORM_CASES = [  # hq, hkv, dh, tokens, with norm
    (4, 4, 64, 1, True), (4, 4, 64, 37, False), (8, 2, 64, 130, True), (28, 4, 128, 1, True), (28, 4, 128, 75, True),
    (6, 2, 128, 400, False), (32, 32, 128, 9, True), (28, 4, 128, 6000, True)]


@pytest.mark.parametrize("hq,hkv,dh,M,norm", NORM_CASES)
def test_norm_rope_into_the_bf16_cache(B, hq, hkv, dh, M, norm):
    rng = np.random.default_rng(hq * 1000 + M)
    rows, max_pos = 2 * M + 3, 2000
    qkv = bf16(rng.normal(size=(M, (hq + 2 * hkv) * dh)) * 2.0 ** rng.integers(-6, 6, (M, 1)))
    gq, gk = bf16(1 + 0.1 * rng.normal(size=dh)), bf16(1 + 0.1 * rng.normal(size=dh))
    pos = rng.integers(0, max_pos, M)
    kv = rng.permutation(rows)[:M]
    if M > 3:
        kv[M // 2] = -1                                   # belongs to no row
        pos[0] = max_pos - 1
    kc0, vc0 = bf16(rng.normal(size=(rows, hkv, dh))), bf16(rng.normal(size=(rows, hkv, dh)))
    kc, vc = kc0.cuda(), vc0.cuda()
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    q0 = bf16(rng.normal(size=(M, hq * dh + 8)))
    q_out = q0.cuda()                                     # rows wider than the queries
    table = B.rope_table(max_pos, dh, THETA)
    args = (gq.cuda() if norm else None, gk.cuda() if norm else None, EPS, ints(pos), ints(kv))
    qd = qkv.cuda()
    got = B.op_qk_norm_rope_kv(qd, *args, kc, vc, hq, hkv, dh, table, q_out=q_out, error_flag=flag)
    assert got is q_out and int(flag.item()) == 0
    x = host(qkv).reshape(M, hq + 2 * hkv, dh)
    q = K.norm_rope(x[:, :hq], host(gq) if norm else None, EPS, pos, THETA)
    k = K.norm_rope(x[:, hq:hq + hkv], host(gk) if norm else None, EPS, pos, THETA)
    live = kv >= 0
    gotq = host(q_out)
    assert (gotq[:, hq * dh:] == host(q0)[:, hq * dh:]).all() and (gotq[~live] == host(q0)[~live]).all()
    # rounding: half a bf16 step of the exact value, taken at the value the kernel may have had before rounding
    tol = lambda y: np.abs(y) * HALF_BF16 + chain_tol(y, dh) * (1 + HALF_BF16) + 1e-38   # noqa: E731
    gq_ = gotq[:, :hq * dh].reshape(M, hq, dh)
    assert (np.abs(gq_ - q)[live] <= tol(q)[live]).all()
    kch, vch = host(kc), host(vc)
    assert (np.abs(kch[kv[live]] - k[live]) <= tol(k)[live]).all()
    assert (vch[kv[live]] == x[live][:, hq + hkv:]).all()
    other = np.setdiff1d(np.arange(rows), kv[live])
    assert (kch[other] == host(kc0)[other]).all() and (vch[other] == host(vc0)[other]).all()
    # in place, and the same bits again
    kc2, vc2 = kc0.cuda(), vc0.cuda()
    inplace = B.op_qk_norm_rope_kv(qd, *args, kc2, vc2, hq, hkv, dh, table, q_out=qd)
    assert inplace is qd and torch.equal(qd[torch.from_numpy(live).cuda()][:, :hq * dh], q_out[torch.from_numpy(live).cuda()][:, :hq * dh])
    assert torch.equal(qd[:, hq * dh:].cpu(), qkv[:, hq * dh:]) and torch.equal(kc2, kc) and torch.equal(vc2, vc)


def test_norm_of_zero_and_of_far_positions(B):
    hq, hkv, dh, max_pos = 2, 1, 128, 200000
    table = B.rope_table(max_pos, dh, 1e6)
    qkv = bf16(np.random.default_rng(0).normal(size=(3, 4 * dh)))
    qkv[0] = 0
    pos = np.array([5, 199999, 131071])
    g = bf16(np.ones(dh)).cuda()
    kc = torch.zeros(3, 1, dh, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    q = host(B.op_qk_norm_rope_kv(qkv.cuda(), g, g, EPS, ints(pos), ints([0, 1, 2]), kc, vc, hq, hkv, dh, table)).reshape(3, 2, dh)
    ref = K.norm_rope(host(qkv).reshape(3, 4, dh)[:, :2], np.ones(dh), EPS, pos, 1e6)
    assert (q[0] == 0).all()
    assert (np.abs(q - ref) <= np.abs(ref) * HALF_BF16 + 2 * chain_tol(ref, dh)).all()


def test_bad_indices_are_skipped_and_flagged(B):
    """Positions, cache rows and spans outside the stated sizes: checked on the device, nothing else is disturbed."""
    hq, hkv, dh, M = 4, 2, 64, 6
    rng = np.random.default_rng(3)
    qkv = bf16(rng.normal(size=(M, (hq + 2 * hkv) * dh))).cuda()
    g = bf16(np.ones(dh)).cuda()
    table = B.rope_table(50, dh, THETA)
    kc = torch.full((8, hkv, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    vc = kc.clone()
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    q_out = torch.full((M, hq * dh), 9.0, dtype=torch.bfloat16, device="cuda")
    B.op_qk_norm_rope_kv(qkv, g, g, EPS, ints([0, 50, -1, 3, 4, 5]), ints([0, 1, 2, 8, 1 << 30, 3]), kc, vc, hq, hkv, dh, table,
                         q_out=q_out, error_flag=flag)
    assert int(flag.item()) >= 100
    assert ((q_out == 9.0).all(1).cpu().numpy() == [False, True, True, True, True, False]).all()
    assert (kc[[1, 2, 4, 5, 6, 7]] == 7.0).all() and not (kc[0] == 7.0).all() and not (vc[3] == 7.0).all()
    # spans: slab not on a block, before the cache, behind it, position behind it; the last row is fine
    codes, scales = random_cache(rng, 4, hkv, dh)
    k8, ks = to_gpu(codes, scales)
    v8, vs = k8.clone(), ks.clone()
    flag.zero_()
    cu, base, at = ints([0, 1, 2, 3, 4, 5, 6]), ints([16, -32, 128, 64, 0, 32]), ints([0, 0, 0, 64, -1, 2])
    B.op_qk_norm_rope_kv8(qkv, g, g, EPS, ints([0, 1, 2, 3, 4, 5]), cu, base, at, ints([0] * 6), k8, v8, ks, vs, hq, hkv, dh,
                          table, q_out=q_out, error_flag=flag)
    assert int(flag.item()) >= 100
    now = k8.view(torch.uint8).cpu().numpy()
    same = (now == codes).all((1, 3))
    assert same.sum() == 4 * 32 - 1 and not same[1, 2]
    flag.zero_()
    ko, _ = B.op_kv8_read(k8, v8, ks, vs, ints([0, 2, 3]), ints([32, 96]), ints([0, 40]), 3,
                          k_out=torch.full((3, hkv, dh), 5.0, dtype=torch.bfloat16, device="cuda"), error_flag=flag)
    assert int(flag.item()) >= 100 and (ko[2] == 5.0).all() and not (ko[0] == 5.0).all()
    flag.zero_()
    out = torch.full((M, hq * dh), 3.0, dtype=torch.bfloat16, device="cuda")
    B.op_attention_kv8(q_out, k8, v8, ks, vs, cu, base, ints([5, 5, 5, 100, -1, 5]), hq, out=out, error_flag=flag)
    assert int(flag.item()) >= 100
    assert ((out == 3.0).all(1).cpu().numpy() == [True, True, True, True, True, False]).all()
    assert torch.isfinite(out[5].float()).all()


WRITE_CASES = [  # hq, hkv, dh, rows of (n, at, had)
    (4, 4, 64, [(1, 0, 0)]),
    (4, 4, 64, [(1, 31, 31), (1, 32, 32), (0, 5, 5), (1, 63, 63), (1, 7, 40)]),           # appends and a rewrite
    (28, 4, 128, [(32, 17, 300), (32, 64, 96), (17, 200, 217), (32, 0, 32), (32, 31, 31)]),   # block steps
    (8, 2, 64, [(100, 0, 0), (33, 0, 0), (31, 0, 31), (64, 30, 200)]),
    (6, 2, 128, [(5, 40, 10), (3, 100, 20)]),                                             # a gap that holds nothing
    (32, 32, 128, [(70, 3, 80), (1, 0, 1)]),
    (28, 4, 128, [(1, int(i * 7 % 130), int(i * 7 % 130)) for i in range(200)])]


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("hq,hkv,dh,rows", WRITE_CASES)
def test_write_into_the_8_bit_cache(B, hq, hkv, dh, rows, norm):
    rng = np.random.default_rng(len(rows) * 10 + dh + norm)
    n, at, had = (np.array(x) for x in zip(*rows))
    base, blocks = slabs(rng, np.maximum(had, at + n))
    M, cu = int(n.sum()), prefix(n)
    pad = 3                                                # tokens behind the last row
    qkv = bf16(rng.normal(size=(M + pad, (hq + 2 * hkv) * dh)) * 2.0 ** rng.integers(-3, 4, (M + pad, 1)))
    gq, gk = bf16(1 + 0.1 * rng.normal(size=dh)), bf16(1 + 0.1 * rng.normal(size=dh))
    row = np.repeat(np.arange(len(n)), n)
    pos = np.concatenate([at[row] + np.arange(M) - cu[row], np.full(pad, 1 << 30)])
    ck, sk = random_cache(rng, blocks, hkv, dh)
    cv, sv = random_cache(rng, blocks, hkv, dh)
    # positions that hold nothing: NaN codes that must neither count nor change
    free = np.ones((blocks * 32,), bool)
    for i in range(len(n)):
        free[base[i]:base[i] + had[i]] = False
    fb = np.nonzero(free)[0]
    ck[fb // 32, :, fb % 32] = 127
    cv[fb // 32, :, fb % 32] = 255
    (k8, ks), (v8, vs) = to_gpu(ck, sk), to_gpu(cv, sv)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    q_out = torch.full((M + pad, hq * dh), 9.0, dtype=torch.bfloat16, device="cuda")
    table = B.rope_table(1000, dh, THETA)

    def run():
        B.op_qk_norm_rope_kv8(qkv.cuda(), gq.cuda() if norm else None, gk.cuda() if norm else None, EPS, ints(pos), ints(cu),
                              ints(base), ints(at), ints(had), k8, v8, ks, vs, hq, hkv, dh, table, q_out=q_out,
                              error_flag=flag)
    run()
    assert int(flag.item()) == 0
    x = host(qkv)[:M].reshape(M, hq + 2 * hkv, dh)
    q = K.norm_rope(x[:, :hq], host(gq) if norm else None, EPS, pos[:M], THETA)
    k = K.norm_rope(x[:, hq:hq + hkv], host(gk) if norm else None, EPS, pos[:M], THETA)
    got = host(q_out)
    assert (got[M:] == 9.0).all()
    assert (np.abs(got[:M].reshape(M, hq, dh) - q) <= np.abs(q) * HALF_BF16 + 2 * chain_tol(q, dh)).all()
    plan = list(zip(cu[:-1], n, base, at, had))
    # V: no arithmetic before the rounding, so codes and scales are the oracle's bit for bit
    rv, rsv = K.write(cv, sv, plan, x[:, hq + hkv:])
    assert (vs.cpu().numpy() == rsv).all() and (v8.view(torch.uint8).cpu().numpy() == rv).all()
    # K: the fp32 chain precedes the rounding.  Scales equal unless the largest magnitude is within the chain's error of
    # 448 2^k; new rows within half an e4m3 step of the exact value; kept rows exactly the oracle's for the scale found.
    rk, rsk = K.write(ck, sk, plan, k)
    gk8, gks = k8.view(torch.uint8).cpu().numpy(), ks.cpu().numpy().astype(np.float64)
    assert (gks == rsk).mean() > 0.999 and (np.abs(np.log2(gks / rsk)) <= 1).all()
    fresh = np.zeros((blocks * 32,), bool)
    exact = np.zeros((blocks * 32, hkv, dh))
    for t0, nn, bb, a, _ in plan:
        fresh[bb + a:bb + a + nn] = True
        exact[bb + a:bb + a + nn] = k[t0:t0 + nn]
    fi = np.nonzero(fresh)[0]
    vals = K.decode(gk8[fi // 32, :, fi % 32]) * gks[fi // 32][..., None]
    want = exact[fi]
    slack = chain_tol(want, dh)
    assert (np.abs(vals - want) <= np.maximum(np.abs(want) * 2.0 ** -4, gks[fi // 32][..., None] * 2.0 ** -10) + 2 * slack).all()
    ki = np.nonzero(~fresh)[0]
    same = (gks == rsk)[ki // 32]
    assert (gk8[ki // 32, :, ki % 32][same] == rk[ki // 32, :, ki % 32][same]).all()
    # a second pass finds everything in place
    before = [t.clone() for t in (k8.view(torch.uint8), v8.view(torch.uint8), ks, vs)]
    run()
    for a, b in zip(before, (k8.view(torch.uint8), v8.view(torch.uint8), ks, vs)):
        assert torch.equal(a, b)


def test_write_borders_of_the_scale_and_what_is_not_finite(B):
    """V (stored without arithmetic): largest magnitudes on and beside 448 2^k, zeros, values under and over the scale's
    range, infinities and NaN."""
    dh, hkv = 64, 1
    tops = [448.0, 450.0, 446.0, 224.0, 226.0, 0.0, 2.0 ** -60, 2.0 ** -31, 2.0 ** 60, 3e38, 1.0, 7.0, 1.75]
    M = len(tops)
    v = np.zeros((M, dh), np.float32)
    for i, t in enumerate(tops):
        v[i] = np.linspace(-t, t, dh)
    v = bf16(v)
    v[-1, 3], v[-1, 4], v[-1, 5] = float("inf"), float("-inf"), float("nan")
    qkv = torch.zeros(M, 3 * dh, dtype=torch.bfloat16)
    qkv[:, 2 * dh:] = v
    k8, v8, ks, vs = B.kv8_cache(32 * M, hkv, dh)
    for t in (k8, v8):
        t.view(torch.uint8).fill_(127)
    ks.fill_(float("nan")), vs.fill_(float("nan"))
    B.op_qk_norm_rope_kv8(qkv.cuda(), None, None, EPS, ints(np.zeros(M)), ints(np.arange(M + 1)), ints(np.arange(M) * 32),
                          ints(np.zeros(M)), ints(np.zeros(M)), k8, v8, ks, vs, 1, 1, dh, B.rope_table(1, dh, THETA))
    ref = host(v)
    for i in range(M):
        mag = np.abs(ref[i])
        k = K.scale_exponent(mag[np.isfinite(mag)].max())
        assert float(vs[i, 0]) == 2.0 ** k, i
        code = v8.view(torch.uint8)[i, 0, 0].cpu().numpy()
        assert (code & 127 == 127).sum() == np.isnan(ref[i]).sum()
        ok = ~np.isnan(ref[i])
        assert (code[ok] == K.encode(ref[i][ok] / 2.0 ** k)).all(), i
    assert (ks.cpu().numpy() == 2.0 ** -40).all() and (k8.view(torch.uint8)[:, 0, 0] & 127 == 0).all()


READ_CASES = [(4, 64, [(33, 0), (1, 31), (0, 0), (160, 5)]), (2, 128, [(7, 30)]), (32, 128, [(100, 0), (31, 1)]),
              (4, 128, [(1, i) for i in range(70)])]


@pytest.mark.parametrize("hkv,dh,rows", READ_CASES)
def test_read_back(B, hkv, dh, rows):
    rng = np.random.default_rng(hkv + dh)
    n, at = (np.array(x) for x in zip(*rows))
    base, blocks = slabs(rng, n + at)
    ck, sk = random_cache(rng, blocks, hkv, dh, spread=33)
    cv, sv = random_cache(rng, blocks, hkv, dh)
    ck[:, :, 3, 5] = 127                                   # a NaN is read as one
    (k8, ks), (v8, vs) = to_gpu(ck, sk), to_gpu(cv, sv)
    total = int(n.sum())
    buf = torch.full((total + 2, hkv, dh), 4.0, dtype=torch.bfloat16, device="cuda")
    ko, vo = B.op_kv8_read(k8, v8, ks, vs, ints(prefix(n)), ints(base), ints(at), total + 2, k_out=buf)
    assert ko is buf and (buf[total:] == 4.0).all()
    kref = np.concatenate([K.span(ck, sk, base[i], at[i], n[i]) for i in range(len(n))])
    vref = np.concatenate([K.span(cv, sv, base[i], at[i], n[i]) for i in range(len(n))])
    assert np.array_equal(host(ko)[:total], kref, equal_nan=True)          # exact: 4 significant bits times 2^k
    assert np.array_equal(host(vo)[:total], vref, equal_nan=True)


ATTN_CASES = [  # hq, hkv, dh, rows of (queries, vis)
    (4, 4, 64, [(1, 1), (1, 31), (1, 32), (1, 33), (0, 50), (1, 0), (1, 159)]),
    (28, 4, 128, [(1, 300), (1, 1), (1, 64), (1, 0), (1, 1111)]),
    (28, 4, 128, [(1, 3000)]),                             # one item per head: its keys over many CTAs
    (32, 32, 128, [(32, 129), (5, 40), (32, 500)]),
    (28, 4, 128, [(32, 300), (32, 96), (0, 10), (17, 64), (32, 0), (70, 70)]),
    (8, 2, 64, [(70, 200), (32, 64), (33, 33), (1, 77)]),
    (6, 2, 128, [(130, 130), (8, 8), (2, 513)]),
    (16, 1, 128, [(1, 90), (3, 1000)]),                    # sixteen and thirty-two query heads on one kv head
    (32, 1, 64, [(2, 100), (1, 33)]),
    (8, 8, 128, [(300, 300), (64, 517), (129, 129), (200, 0)]),
    (4, 2, 128, [(2, int(i * 37 % 400)) for i in range(150)]),
    (28, 4, 128, [(400, 400), (250, 900), (1, 333)]),
    # steps long enough for every variant: whole rows of several query tiles beside short rows and an empty one
    (16, 2, 128, [(260, 260), (32, 1500), (0, 0), (40, 130)]),
]


def attn_inputs(rng, hq, hkv, dh, rows, spread=4, qscale=1.0):
    n, vis = (np.array(x) for x in zip(*rows))
    base, blocks = slabs(rng, vis)
    ck, sk = random_cache(rng, blocks, hkv, dh, spread=0)
    sk = sk * 2.0 ** rng.integers(-3, 2, sk.shape)
    cv, sv = random_cache(rng, blocks, hkv, dh, spread=spread)
    unseen = np.ones(blocks * 32, bool)
    for i in range(len(n)):
        unseen[base[i]:base[i] + vis[i]] = False
    u = np.nonzero(unseen)[0]
    ck[u // 32, :, u % 32], cv[u // 32, :, u % 32] = 127, 255      # NaN everywhere a row does not see
    blank = unseen.reshape(blocks, 32).all(1)
    sk[blank], sv[blank] = np.nan, np.inf
    M = int(n.sum())
    q = bf16(rng.normal(size=(M, hq * dh)) * qscale * 2.0 ** rng.integers(-2, 2, (M, 1)))
    return n, vis, base, (ck, sk), (cv, sv), q


def attn_bound(out, mag, dot, flat, vmax, n_keys, dh):
    """How far a correct kernel may be: the output's rounding to bf16; a query element held to 2^-17 of its row's largest
    element at worst (as two e4m3 values: the largest lies in [2^7, 2^8), half the second value's least step is 2^-10);
    scores in fp32 (dh products, a relative 2^-23 per accumulation, the scale and the base-2 exponent's argument 4 more),
    their error e^d - 1 on every weight; weights rounded to fp16 (2^-11, or half the subnormal step, 2^-25, where the
    largest weight is 2^2 at least), exponentials 2^-21; fp32 sums over the keys in chunks of 16."""
    d = dot * (dh + 4) * 2.0 ** -23 + flat * 2.0 ** -17
    w = np.expm1(2 * d) + 2.0 ** -11 + 2.0 ** -20 + (n_keys / 16 + 16) * 2.0 ** -23
    return (np.abs(out) * HALF_BF16 + mag * w + n_keys * 2.0 ** -27 * vmax) * (1 + 2.0 ** -7) + 1e-37


def check_attention(got, q, hq, dh, n, vis, base, kc, vc):
    cu = prefix(n)
    for i in range(len(n)):
        if n[i] == 0:
            continue
        g = got[cu[i]:cu[i + 1]].reshape(n[i], hq, dh)
        if vis[i] == 0:
            assert (g == 0).all(), f"row {i} sees nothing"
            continue
        k, v = K.span(*kc, base[i], 0, vis[i]), K.span(*vc, base[i], 0, vis[i])
        ref, mag, dot, flat = K.attention(host(q)[cu[i]:cu[i + 1]].reshape(n[i], hq, dh), k, v)
        err, tol = np.abs(g - ref), attn_bound(ref, mag, dot, flat, np.abs(v).max(), vis[i], dh)
        assert (err <= tol).all(), f"row {i}: error {err.max()} at most {(err / tol).max()} of the bound"


@pytest.mark.parametrize("hint", ["exact", "unknown"])
@pytest.mark.parametrize("hq,hkv,dh,rows", ATTN_CASES)
def test_attention_over_the_8_bit_cache(B, hq, hkv, dh, rows, hint):
    rng = np.random.default_rng(hq * 31 + len(rows))
    n, vis, base, kc, vc, q = attn_inputs(rng, hq, hkv, dh, rows)
    (k8, ks), (v8, vs) = to_gpu(*kc), to_gpu(*vc)
    M, pad = int(n.sum()), 2
    qd = torch.cat([q, torch.full((pad, hq * dh), float("nan"), dtype=torch.bfloat16)]).cuda()
    out = torch.full((M + pad, hq * dh), 6.0, dtype=torch.bfloat16, device="cuda")
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    kw = dict(max_nq=int(n.max()), max_vis=int(vis.max())) if hint == "exact" else {}
    run = lambda o: B.op_attention_kv8(qd, k8, v8, ks, vs, ints(prefix(n)), ints(base), ints(vis), hq, out=o,   # noqa: E731
                                       error_flag=flag, **kw)
    run(out)
    assert int(flag.item()) == 0
    assert (out[M:] == 6.0).all()                          # rows behind the last sequence are left as they were
    check_attention(host(out)[:M], q, hq, dh, n, vis, base, kc, vc)
    again = torch.full_like(out, 6.0)
    run(again)
    assert torch.equal(again, out)                         # the same bits every time


@pytest.mark.parametrize("hq,hkv,dh,rows", [(4, 4, 64, [(1, 200), (3, 70)]), (28, 4, 128, [(32, 500), (1, 900)]),
                                            (32, 32, 128, [(1, 640)]), (28, 4, 128, [(300, 300)])])
def test_attention_with_scales_far_apart(B, hq, hkv, dh, rows):
    """V blocks whose scales differ by up to 2^56, so that one accumulator meets very large and very small values."""
    rng = np.random.default_rng(dh + len(rows))
    n, vis, base, kc, vc, q = attn_inputs(rng, hq, hkv, dh, rows, spread=28, qscale=0.05)
    (k8, ks), (v8, vs) = to_gpu(*kc), to_gpu(*vc)
    out = B.op_attention_kv8(q.cuda(), k8, v8, ks, vs, ints(prefix(n)), ints(base), ints(vis), hq, max_nq=int(n.max()))
    check_attention(host(out), q, hq, dh, n, vis, base, kc, vc)


@pytest.mark.parametrize("hq,hkv,nq", [(28, 4, 1), (28, 4, 32), (32, 32, 1), (32, 32, 32)])
def test_attention_weights_on_small_scaled_values(B, hq, hkv, nq):
    """The keys that win hold tiny values beside blocks of huge ones that get almost no weight."""
    rng = np.random.default_rng(nq + hq)
    dh, vis = 128, 320
    n, vis, base, kc, vc, q = attn_inputs(rng, hq, hkv, dh, [(nq, vis)], spread=0)
    ck, sk = kc
    ck[:] = rng.integers(0, 40, ck.shape)
    win = base[0] // 32 + 4
    q[:] = bf16(np.abs(rng.normal(size=q.shape)) + 0.5)
    ck[win] = 100                                          # large positive keys against positive queries
    sk[:] = 2.0 ** -3
    vc[1][:] = 2.0 ** 10
    vc[1][win] = 2.0 ** -14
    (k8, ks), (v8, vs) = to_gpu(ck, sk), to_gpu(*vc)
    out = B.op_attention_kv8(q.cuda(), k8, v8, ks, vs, ints([0, nq]), ints(base), ints(vis), hq, max_nq=nq, max_vis=320)
    check_attention(host(out), q, hq, dh, n, vis, base, (ck, sk), vc)


def test_attention_reads_queries_of_a_qkv_buffer(B):
    rng = np.random.default_rng(5)
    hq, hkv, dh = 28, 4, 128
    n, vis, base, kc, vc, q = attn_inputs(rng, hq, hkv, dh, [(9, 100), (32, 64)])
    (k8, ks), (v8, vs) = to_gpu(*kc), to_gpu(*vc)
    qkv = torch.full((41, (hq + 2 * hkv) * dh), float("nan"), dtype=torch.bfloat16, device="cuda")
    qkv[:, :hq * dh] = q.cuda()
    a = (k8, v8, ks, vs, ints(prefix(n)), ints(base), ints(vis), hq)
    assert torch.equal(B.op_attention_kv8(qkv, *a, max_nq=32), B.op_attention_kv8(q.cuda(), *a, max_nq=32))
    assert torch.equal(B.op_attention_kv8(qkv[:, :hq * dh], *a, max_nq=32), B.op_attention_kv8(q.cuda(), *a, max_nq=32))


def test_attention_of_queries_that_are_not_finite(B):
    """A NaN query gives NaN in its own head's output and nowhere else; a zero query averages."""
    rng = np.random.default_rng(6)
    for nq in (1, 40):
        hq, hkv, dh = 14, 2, 128
        n, vis, base, kc, vc, q = attn_inputs(rng, hq, hkv, dh, [(nq, 90)])
        q[0, :dh] = float("nan")
        q[0, dh:2 * dh] = 0
        (k8, ks), (v8, vs) = to_gpu(*kc), to_gpu(*vc)
        got = host(B.op_attention_kv8(q.cuda(), k8, v8, ks, vs, ints([0, nq]), ints(base), ints(vis), hq, max_nq=nq))
        got = got.reshape(nq, hq, dh)
        assert np.isnan(got[0, 0]).all() and np.isfinite(got[0, 1:]).all() and np.isfinite(got[1:]).all()
        mean = K.span(*vc, base[0], 0, 90)[:, 0].mean(0)
        assert (np.abs(got[0, 1] - mean) <= np.abs(mean) * HALF_BF16 + np.abs(K.span(*vc, base[0], 0, 90)).max() * 2.0 ** -11).all()


@pytest.mark.parametrize("nq", [1, 32, 64])
def test_offsets_beyond_32_bits(B, nq):
    """A cache of more than 4 GiB of codes: rows near its end, written, attended to and read back."""
    hq, hkv, dh = 32, 32, 128
    blocks = (1 << 32) // (hkv * 32 * dh) + 60
    k8, v8, ks, vs = B.kv8_cache(blocks * 32, hkv, dh)
    assert k8.numel() > 1 << 32
    rng = np.random.default_rng(nq)
    at, base = 61, (blocks - 5) * 32
    M = at + nq
    qkv = bf16(rng.normal(size=(M, 3 * hq * dh)))
    table = B.rope_table(200, dh, THETA)
    g = bf16(np.ones(dh)).cuda()
    args = lambda s, a, h, c: (qkv[s].cuda(), g, g, EPS, ints(np.arange(M)[s]), ints([0, c]), ints([base]), ints([a]), ints([h]),   # noqa: E731
                               k8, v8, ks, vs, hq, hkv, dh, table)
    B.op_qk_norm_rope_kv8(*args(slice(0, at), 0, 0, at))
    q = B.op_qk_norm_rope_kv8(*args(slice(at, M), at, at, nq))
    ko, vo = B.op_kv8_read(k8, v8, ks, vs, ints([0, M]), ints([base]), ints([0]), M)
    out = B.op_attention_kv8(q, k8, v8, ks, vs, ints([0, nq]), ints([base]), ints([M]), hq, max_nq=nq)
    k, v = host(ko), host(vo)
    x = host(qkv).reshape(M, 3 * hq, dh)
    # the scale of a block can be twice what a value alone would need: half a step of e4m3, or half a subnormal step
    top = np.abs(x[:, 64:]).max()
    assert (np.abs(v - x[:, 64:]) <= np.maximum(np.abs(x[:, 64:]) * 2.0 ** -4, top / 224 * 2.0 ** -10)).all()
    ref, mag, dot, flat = K.attention(host(q).reshape(nq, hq, dh), k, v)
    assert (np.abs(host(out).reshape(nq, hq, dh) - ref) <= attn_bound(ref, mag, dot, flat, np.abs(v).max(), M, dh)).all()


def test_a_step_of_serving(B):
    """The operators as they are used: whole prompts into both caches, then block steps and single tokens that rewrite and
    append, attention after every write.  The 8-bit path is followed exactly on what it read back, and stays near the
    bf16 path (whose kernels are the framework's own)."""
    hq, hkv, dh = 28, 4, 128
    rng = np.random.default_rng(11)
    p = np.array([70, 33, 128])
    total = p + 40
    base, blocks = slabs(rng, total)
    cache = B.kv8_cache(blocks * 32, hkv, dh)
    for t in cache[:2]:
        t.view(torch.uint8).fill_(127)
    kc = torch.zeros(blocks * 32, hkv, dh, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    table = B.rope_table(256, dh, THETA)
    g = [bf16(1 + 0.1 * rng.normal(size=dh)).cuda() for _ in range(2)]
    length = np.zeros(3, np.int64)
    steps = [("whole", np.zeros(3, np.int64), p), ("block", p, np.array([32, 32, 32])), ("rewrite", p, np.array([32, 32, 32])),
             ("token", p + 32, np.ones(3, np.int64)), ("token", p + 33, np.ones(3, np.int64))]
    scratch = B.attention_kv8_scratch(hq, hkv, dh)
    for name, at, n in steps:
        M, cu = int(n.sum()), prefix(n)
        row = np.repeat(np.arange(3), n)
        pos = at[row] + np.arange(M) - cu[row]
        qkv = bf16(rng.normal(size=(M, (hq + 2 * hkv) * dh))).cuda()
        had, length = length, np.maximum(length, at + n)
        q8 = B.op_qk_norm_rope_kv8(qkv, *g, EPS, ints(pos), ints(cu), ints(base), ints(at), ints(had), *cache, hq, hkv, dh, table)
        o8 = B.op_attention_kv8(q8, *cache, ints(cu), ints(base), ints(length), hq, max_nq=int(n.max()),
                                max_vis=int(length.max()), scratch=scratch)
        q16 = B.op_qk_norm_rope_kv(qkv, *g, EPS, ints(pos), ints(base[row] + pos), kc, vc, hq, hkv, dh, table)
        assert torch.equal(q8, q16)
        buf = torch.empty(M, (hq + 2 * hkv) * dh, dtype=torch.bfloat16, device="cuda")
        buf[:, :hq * dh] = q16
        o16 = B.op_attention(buf, kc, vc, ints(cu), ints(base), ints(length), hq, hkv, dh)
        k, v = (host(t) for t in B.op_kv8_read(*cache, ints(prefix(length)), ints(base), ints(np.zeros(3)), int(length.sum())))
        got, at_row = host(o8), prefix(length)
        for i in range(3):
            ki, vi = k[at_row[i]:at_row[i + 1]], v[at_row[i]:at_row[i + 1]]
            ref, mag, dot, flat = K.attention(host(q8)[cu[i]:cu[i + 1]].reshape(-1, hq, dh), ki, vi)
            err = np.abs(got[cu[i]:cu[i + 1]].reshape(-1, hq, dh) - ref)
            assert (err <= attn_bound(ref, mag, dot, flat, np.abs(vi).max(), len(ki), dh)).all(), (name, i)
        # 8 bits move a key's dims by at most 2^-4 of themselves, in all directions: the outputs stay alike
        a, b = got, host(o16)
        assert np.linalg.norm(a - b) < 0.1 * np.linalg.norm(b), name


def test_captured_and_replayed(B):
    """Write + attention of two layers captured into two graphs (own scratch each), replayed with new inputs, on another
    stream, against eager calls."""
    hq, hkv, dh = 28, 4, 128
    rng = np.random.default_rng(12)
    n, had = np.array([32, 1, 32, 5]), np.array([100, 64, 0, 31])
    base, blocks = slabs(rng, had + n)
    M, cu = int(n.sum()), prefix(n)
    row = np.repeat(np.arange(4), n)
    pos = ints(had[row] + np.arange(M) - cu[row])
    table = B.rope_table(256, dh, THETA)
    g = bf16(np.ones(dh)).cuda()
    qkv = torch.empty(M, (hq + 2 * hkv) * dh, dtype=torch.bfloat16, device="cuda")
    cu_d, base_d, had_d, vis_d = ints(cu), ints(base), ints(had), ints(had + n)
    caches = []
    for layer in range(2):
        ck, sk = random_cache(rng, blocks, hkv, dh)
        cv, sv = random_cache(rng, blocks, hkv, dh)
        (k8, ks), (v8, vs) = to_gpu(ck, sk), to_gpu(cv, sv)
        caches.append((k8, v8, ks, vs))
    start = [[t.clone() for t in c] for c in caches]

    def step(c):
        q = B.op_qk_norm_rope_kv8(qkv, g, g, EPS, pos, cu_d, base_d, had_d, had_d, *c, hq, hkv, dh, table)
        return B.op_attention_kv8(q, *c, cu_d, base_d, vis_d, hq, max_nq=32, max_vis=int((had + n).max()))

    def reset():
        for c, s in zip(caches, start):
            for a, b in zip(c, s):
                a.view(torch.uint8).copy_(b.view(torch.uint8)) if a.dtype == torch.float8_e4m3fn else a.copy_(b)

    inputs = [bf16(rng.normal(size=qkv.shape)).cuda() for _ in range(2)]
    want = []
    for x in inputs:
        reset()
        qkv.copy_(x)
        want.append([step(c).clone() for c in caches])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(side):
        for c in caches:
            gr = torch.cuda.CUDAGraph()
            with torch.cuda.graph(gr, stream=side):
                out = step(c)
            graphs.append((gr, out))
        for x, w in zip(inputs, want):
            reset()
            qkv.copy_(x)
            for gr, _ in graphs:
                gr.replay()
            side.synchronize()
            for (_, out), ref in zip(graphs, w):
                assert torch.equal(out, ref)
    torch.cuda.current_stream().wait_stream(side)


def test_two_streams_at_once(B):
    """Independent calls on two streams, each with scratch of its own, give what they give alone."""
    hq, hkv, dh = 32, 32, 128
    sets, want = [], []
    for seed in (1, 2):
        rng = np.random.default_rng(seed)
        n, vis, base, kc, vc, q = attn_inputs(rng, hq, hkv, dh, [(1, 2000 + seed), (1, 900), (1, 50)])
        a = (q.cuda(), *(t for pair in zip(to_gpu(*kc), to_gpu(*vc)) for t in pair), ints(prefix(n)), ints(base), ints(vis), hq)
        sets.append(a)
        want.append(B.op_attention_kv8(*a, max_nq=1))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    outs = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                outs[i].append(B.op_attention_kv8(*sets[i], max_nq=1))
    torch.cuda.synchronize()
    for i in range(2):
        for o in outs[i]:
            assert torch.equal(o, want[i])


HINT_CASES = [  # hq, hkv, dh, rows of (queries, vis): one token a row, block steps, long and short rows mixed, whole rows
    (28, 4, 128, [(1, 40), (1, 2500), (1, 0), (1, 129)]),
    (8, 8, 64, [(32, 96), (5, 700), (0, 9), (32, 0), (1, 33)]),
    (32, 32, 128, [(32, 64)] * 20 + [(32, 600), (2, 1)]),
    (14, 2, 128, [(70, 300), (3, 31), (129, 1200)])]


@pytest.mark.parametrize("max_nq,max_vis", [(0, 0), (1, 1), (0, 1), (1, 0), (3, 128), (1 << 20, 1 << 20)])
@pytest.mark.parametrize("hq,hkv,dh,rows", HINT_CASES)
def test_hints_choose_the_kernel_and_nothing_else(B, hq, hkv, dh, rows, max_nq, max_vis):
    """Too small, too large and absent: rows of any length come out right, and a row that does not fit is skipped alone."""
    rng = np.random.default_rng(len(rows) + dh)
    n, vis, base, kc, vc, q = attn_inputs(rng, hq, hkv, dh, rows)
    (k8, ks), (v8, vs) = to_gpu(*kc), to_gpu(*vc)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full((len(q), hq * dh), 6.0, dtype=torch.bfloat16, device="cuda")
    call = lambda v: B.op_attention_kv8(q.cuda(), k8, v8, ks, vs, ints(prefix(n)), ints(base), ints(v), hq, max_nq=max_nq,   # noqa: E731
                                        max_vis=max_vis, out=out, error_flag=flag)
    call(vis)
    assert int(flag.item()) == 0
    check_attention(host(out), q, hq, dh, n, vis, base, kc, vc)
    out.fill_(6.0)
    wrong = vis.copy()
    wrong[1] = k8.shape[0] * 32 + 1 - base[1]
    call(wrong)
    lo, hi = prefix(n)[1:3]
    assert int(flag.item()) >= 100
    assert (out[lo:hi] == 6.0).all()
    # (not the bits of before: where the rows' keys are split depends on all of them)
    rest = np.arange(len(n)) != 1
    left = np.concatenate([host(out)[:lo], host(out)[hi:]])
    check_attention(left, torch.cat([q[:lo], q[hi:]]), hq, dh, n[rest], vis[rest], base[rest], kc, vc)


@pytest.mark.parametrize("hq,hkv,dh", [(8, 8, 64), (9, 3, 128)])
def test_write_with_several_heads_to_a_block_of_threads(B, hq, hkv, dh):
    """Enough cache blocks that one CTA walks over the kv heads: codes and scales of V bit for bit, K by its scale."""
    rng = np.random.default_rng(dh)
    n = np.full(40, 300) + rng.integers(-40, 40, 40)
    at = rng.integers(0, 64, 40)
    base, blocks = slabs(rng, at + n)
    M, cu = int(n.sum()), prefix(n)
    qkv = bf16(rng.normal(size=(M, (hq + 2 * hkv) * dh)))
    g = bf16(np.ones(dh))
    row = np.repeat(np.arange(len(n)), n)
    pos = at[row] + np.arange(M) - cu[row]
    ck, sk = random_cache(rng, blocks, hkv, dh)
    cv, sv = random_cache(rng, blocks, hkv, dh)
    (k8, ks), (v8, vs) = to_gpu(ck, sk), to_gpu(cv, sv)
    B.op_qk_norm_rope_kv8(qkv.cuda(), g.cuda(), g.cuda(), EPS, ints(pos), ints(cu), ints(base), ints(at), ints(at), k8, v8,
                          ks, vs, hq, hkv, dh, B.rope_table(1000, dh, THETA))
    x = host(qkv).reshape(M, hq + 2 * hkv, dh)
    plan = list(zip(cu[:-1], n, base, at, at))
    rv, rsv = K.write(cv, sv, plan, x[:, hq + hkv:])
    assert (vs.cpu().numpy() == rsv).all() and (v8.view(torch.uint8).cpu().numpy() == rv).all()
    k = K.norm_rope(x[:, hq:hq + hkv], np.ones(dh), EPS, pos, THETA)
    gk8, gks = k8.view(torch.uint8).cpu().numpy(), ks.cpu().numpy().astype(np.float64)
    at_row = base[row] + pos
    vals = K.decode(gk8[at_row // 32, :, at_row % 32]) * gks[at_row // 32][..., None]
    assert (np.abs(vals - k) <= np.maximum(np.abs(k) * 2.0 ** -4, gks[at_row // 32][..., None] * 2.0 ** -10) + 2 * chain_tol(k, dh)).all()


def test_rows_that_stay_keep_their_nan_to_themselves(B):
    """A kept row's NaN codes meet neither the rotation nor the norm of the new rows beside it; its finite codes follow the
    scale."""
    hq, hkv, dh = 2, 2, 64
    rng = np.random.default_rng(11)
    ck, sk = random_cache(rng, 2, hkv, dh)
    ck[1, 0, 3, 7], ck[1, 1, 4, 40] = 127, 255
    (k8, ks), (v8, vs) = to_gpu(ck, sk), to_gpu(ck, sk)
    qkv = bf16(rng.normal(size=(4, 6 * dh)) * 8)
    g = bf16(np.ones(dh)).cuda()
    B.op_qk_norm_rope_kv8(qkv.cuda(), g, g, EPS, ints([5, 6, 7, 8]), ints([0, 4]), ints([32]), ints([5]), ints([5]), k8, v8, ks,
                          vs, hq, hkv, dh, B.rope_table(50, dh, THETA))
    for codes, scales in ((k8, ks), (v8, vs)):
        c, s = codes.view(torch.uint8).cpu().numpy(), scales.cpu().numpy().astype(np.float64)
        was = K.decode(ck[1, :, :5]) * sk[1][:, None, None]
        now = K.decode(c[1, :, :5]) * s[1][:, None, None]
        assert np.array_equal(np.isnan(now), np.isnan(was)) and np.isnan(now).sum() == 2
        half_step = np.maximum(np.abs(was) * 2.0 ** -4, s[1][:, None, None] * 2.0 ** -10)
        assert (np.abs(now - was)[~np.isnan(was)] <= half_step[~np.isnan(was)]).all()
        assert not np.isnan(K.decode(c[1, :, 5:9])).any()


@pytest.mark.parametrize("hq,hkv,dh,rows", [(28, 4, 128, [(32, 9000)]), (8, 2, 64, [(40, 4200), (9, 700), (33, 0)])])
def test_a_few_long_rows_in_many_chunks(B, hq, hkv, dh, rows):
    """Few query tiles over long rows: the keys are cut into as many chunks as the rows' lengths allow, some of them empty."""
    rng = np.random.default_rng(dh)
    n, vis, base, kc, vc, q = attn_inputs(rng, hq, hkv, dh, rows, qscale=0.2)
    (k8, ks), (v8, vs) = to_gpu(*kc), to_gpu(*vc)
    out = B.op_attention_kv8(q.cuda(), k8, v8, ks, vs, ints(prefix(n)), ints(base), ints(vis), hq, max_nq=int(n.max()),
                             max_vis=int(vis.max()))
    check_attention(host(out), q, hq, dh, n, vis, base, kc, vc)


@pytest.mark.parametrize("hq,hkv,dh,nq,vis", [(14, 2, 128, 1, 200), (14, 2, 128, 40, 90), (14, 2, 128, 40, 200), (8, 2, 64, 64, 333),
                                              (28, 4, 128, 600, 700)])
@pytest.mark.parametrize("what", [float("inf"), float("-inf"), float("nan")])
def test_what_is_not_finite_stays_in_its_query_row(B, hq, hkv, dh, nq, vis, what):
    rng = np.random.default_rng(nq)
    n, vis, base, kc, vc, q = attn_inputs(rng, hq, hkv, dh, [(nq, vis)])
    q[0, dh + 5] = what
    (k8, ks), (v8, vs) = to_gpu(*kc), to_gpu(*vc)
    out = host(B.op_attention_kv8(q.cuda(), k8, v8, ks, vs, ints([0, nq]), ints(base), ints(vis), hq, max_nq=nq, max_vis=int(vis[0])))
    out = out.reshape(nq, hq, dh)
    assert np.isnan(out[0, 1]).all()
    out[0, 1] = 0
    assert np.isfinite(out).all()


def some_rows(count, nq, lo, hi, longest):
    """`count` rows of nq queries (a few of fewer, one of none) over lo..hi keys, one over `longest`, one over nothing."""
    rng = np.random.default_rng(count)
    rows = [(nq if i % 7 else max(1, nq - 3), int(v)) for i, v in enumerate(rng.integers(lo, hi + 1, count))]
    rows[1], rows[2], rows[count // 2] = (nq, 0), (0, hi), (nq, longest)
    return rows


WAYS = [  # hq, hkv, dh, rows, whether the largest number of keys is told, scratch expected
    (32, 32, 128, some_rows(32, 9, 1, 200, 300), True, 0),        # single-warp workers, one per item
    (32, 32, 128, some_rows(80, 9, 1, 70, 700), True, 1),         # single-warp workers on the shared line
    (16, 16, 64, some_rows(60, 12, 1, 200, 500), True, 0),
    (16, 16, 64, some_rows(160, 10, 1, 60, 800), True, 1),
    (6, 2, 128, some_rows(6, 4, 1, 900, 2800), False, 1),         # four-warp workers, two query tiles: line, one per item
    (6, 2, 128, some_rows(6, 4, 1, 900, 1800), True, 0),
    (8, 2, 64, some_rows(6, 4, 1, 900, 2800), False, 1),
    (8, 2, 64, some_rows(6, 24, 1, 900, 1800), True, 0),
    (28, 4, 128, some_rows(9, 1, 1, 900, 2800), False, 1),        # one query tile
    (4, 4, 64, some_rows(120, 1, 1, 300, 4000), True, 0),
    (28, 4, 128, some_rows(12, 32, 1, 80, 96), True, 0),          # wide, but brief
    (28, 4, 128, some_rows(5, 40, 100, 400, 1300), True, 1)]      # tensor-core tiles, keys cut


@pytest.mark.parametrize("hq,hkv,dh,rows,told,scratch", WAYS)
def test_every_way_through_the_attention(B, hq, hkv, dh, rows, told, scratch):
    rng = np.random.default_rng(len(rows) + hq)
    n, vis, base, kc, vc, q = attn_inputs(rng, hq, hkv, dh, rows, qscale=0.5)
    (k8, ks), (v8, vs) = to_gpu(*kc), to_gpu(*vc)
    hints = dict(max_nq=int(n.max()), max_vis=int(vis.max()) if told else 0)
    assert B.lib().bs_op_attention_kv8_uses_scratch(len(n), len(q), hints["max_nq"], hints["max_vis"], hq, hkv, dh) == scratch
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    run = lambda: B.op_attention_kv8(q.cuda(), k8, v8, ks, vs, ints(prefix(n)), ints(base), ints(vis), hq, error_flag=flag, **hints)   # noqa: E731
    out = run()
    assert int(flag.item()) == 0
    check_attention(host(out), q, hq, dh, n, vis, base, kc, vc)
    assert torch.equal(out, run())
