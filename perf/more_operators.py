"""Cases of the operators between a hidden state and a committed token: 8-bit integer codes of activations, the
projections over them (with scales for each token and each output channel), and the rules of constrained decoding on
logits - penalties for repeated tokens, biases, grammar masks - applied to the logits themselves or within the
confidence pass.

Shapes are the ones this repository serves: d_model 3584 / 4096, 4608 QKV rows, d_ffn 18944 / 12288, vocabularies of
152064 and 126464 entries, blocks of 32 tokens in batches of 16 and 64 rows; and the small shapes of its tests."""
import math

import numpy as np
import torch

own = False


# ---- cases -------------------------------------------------------------------------------------------------

def listed():
    return [
        # the tokens of a small single-token batch before a projection: latency
        dict(name="quant 16x3584", op="quant", m=16, k=3584, type="bf16", gather=0, mix=1),
        # the SwiGLU outputs of a refresh before the down projection
        dict(name="quant 4096x18944", op="quant", m=4096, k=18944, type="bf16", gather=0, mix=2),
        # QKV projection of a batch of single tokens: weights streamed once
        dict(name="gemm 64 qkv", op="gemm", m=64, n=4608, k=3584, mode=0, mix=3),
        # gate / up of the benchmark's block step
        dict(name="gemm 512 gate/up", op="gemm", m=512, n=18944, k=3584, mode=3, mix=4),
        # down projection of a block-start refresh: bound by arithmetic
        dict(name="gemm 8192 down", op="gemm", m=8192, n=3584, k=18944, mode=0, mix=5),
        # LM head of a small block step: fp32 logits
        dict(name="gemm 128 lm head", op="gemm", m=128, n=152064, k=3584, mode=2, mix=6),
        # the smallest model's single-token rows, all rules
        dict(name="rules 4x1 v1024", op="rules", reqs=4, per=1, v=1024, type="f32", lo=9, hi=160, bias=8, masks=4, rep=1, mix=7),
        # single-token rows of a batch, long contexts, penalties and biases, no grammar
        dict(name="rules 64x1 v152064", op="rules", reqs=64, per=1, v=152064, type="f32", lo=512, hi=4096, bias=100, masks=0,
             rep=1, mix=8),
        # a block step with a grammar, logits in 16 bits
        dict(name="rules 16x32 v126464 bf16", op="rules", reqs=16, per=32, v=126464, type="bf16", lo=320, hi=800, bias=20,
             masks=512, rep=1, mix=9),
        # confidence of four single-token rows: latency
        dict(name="conf 4x1 v152064", op="conf", reqs=4, per=1, v=152064, type="f32", lo=64, hi=1024, bias=16, masks=4, rep=1,
             mix=10),
        # confidence of a batch of single tokens with long contexts
        dict(name="conf 64x1 v126464", op="conf", reqs=64, per=1, v=126464, type="f32", lo=512, hi=4096, bias=100, masks=32,
             rep=1, mix=11),
        # confidence of the benchmark's block step: penalties, biases, a grammar mask for some rows
        dict(name="conf 16x32 v152064", op="conf", reqs=16, per=32, v=152064, type="f32", lo=320, hi=800, bias=20, masks=256,
             rep=1, mix=12),
    ]


# (output features, input features) of the projections of the shapes above; the last ones are the tests' models
PROJECTIONS = [(4608, 3584), (3584, 3584), (18944, 3584), (3584, 18944), (12288, 4096), (4096, 12288), (4096, 4096),
               (704, 256), (1000, 384), (384, 1000), (2000, 384)]
VOCABS = [1024, 2000, 126464, 152064, 152064]


def _log(rng, a, b):
    return max(a, min(b, int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))))


def draw(rng):
    op = rng.choice(["quant", "gemm", "gemm", "gemm", "rules", "conf", "conf"])
    mix = rng.randrange(1 << 20)
    if op == "quant":
        c = dict(op=op, m=_log(rng, 1, 16384), k=rng.choice([256, 384, 3584, 4096, 12288, 18944, _log(rng, 16, 20000)]),
                 type=rng.choice(["bf16", "bf16", "f32"]), gather=int(rng.random() < 0.25), mix=mix)
        dim = "m"
    elif op == "gemm":
        n, k = rng.choice(PROJECTIONS) if rng.random() < 0.7 else (_log(rng, 24, 20000), _log(rng, 32, 20000))
        c = dict(op=op, m=rng.choice([_log(rng, 1, 8192), _log(rng, 1, 1024)]), n=n, k=k, mode=rng.choice([0, 0, 2, 3]), mix=mix)
        dim = "m"
    else:
        v = rng.choice(VOCABS) if rng.random() < 0.75 else _log(rng, 500, 160000)
        hi = _log(rng, 16, 8192)
        per = rng.choice([1, 1, 32, _log(rng, 2, 64)])
        c = dict(op=op, reqs=_log(rng, 1, 96), per=per, v=v, type=rng.choice(["f32", "f32", "bf16"]),
                 lo=max(1, int(hi * rng.uniform(0.02, 1.0))), hi=hi, bias=rng.choice([0, 8, 100, 300]), masks=0,
                 rep=rng.choice([0, 1, 1, 1]), mix=mix)
        dim = "reqs"
        share = rng.choice([0, 0, 1, per])       # no grammar, a mask for each request or for each row
        c["masks"] = c["reqs"] * share
    most = max(_cost(x) for x in listed() if x["op"] == op)
    while c[dim] > 1 and _cost(c) > most:
        c[dim] = max(1, c[dim] * 3 // 4)
        if dim == "reqs":
            c["masks"] = c["reqs"] * share
    return c


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 400)


def _plan(case):
    """Request of each logits row, its context's length and how much of it is prompt, its number of biases, its mask."""
    r = np.random.RandomState(case["mix"])
    reqs = case["reqs"]
    n = np.full(reqs, case["per"]) if case["per"] == 1 else r.randint(max(1, case["per"] // 4), case["per"] + 1, reqs)
    row_req = np.repeat(np.arange(reqs), n)
    ctx = r.randint(case["lo"], case["hi"] + 1, reqs)
    gen = (ctx * r.uniform(0.1, 0.9, reqs)).astype(np.int64)
    bias = np.minimum(r.randint(0, case["bias"] + 1, reqs), case["v"] // 2)
    rows = len(row_req)
    mask = np.where(r.rand(rows) < 0.9, r.permutation(np.arange(rows) % max(1, case["masks"])), -1)
    return dict(rows=rows, row_req=row_req, ctx=ctx, gen=gen, bias=bias, row_mask=mask)


def work(case):
    if case["op"] == "quant":
        m, k = case["m"], case["k"]
        return {"bytes": m * k * (3 if case["type"] == "bf16" else 5) + 4 * m + 4 * m * case["gather"], "flops": 4 * m * k}
    if case["op"] == "gemm":
        m, n, k, two = case["m"], case["n"], case["k"], 1 + (case["mode"] == 3)
        return {"bytes": m * k + 4 * m + two * (n * k + 4 * n) + m * n * (4 if case["mode"] == 2 else 2),
                "flops": 2 * two * m * n * k}
    p, v = _plan(case), case["v"]
    size = 4 if case["type"] == "f32" else 2
    rules = 4 * int(p["ctx"].sum()) * case["rep"] + 8 * int(p["bias"].sum()) + 4 * p["rows"]
    masks = case["masks"] and len(np.unique(p["row_mask"][p["row_mask"] >= 0])) * ((v + 31) // 32) * 4 + 4 * p["rows"]
    if case["op"] == "rules":
        return {"bytes": 2 * p["rows"] * v * size + rules + masks, "flops": 2 * p["rows"] * v}
    return {"bytes": p["rows"] * (v * size + 8) + rules + masks, "flops": 4 * p["rows"] * v}


# ---- inputs ------------------------------------------------------------------------------------------------

def _codes(rows, k, g):
    """int8 codes of normally distributed rows whose largest element has 127 (rows start at multiples of 16 bytes)."""
    store = torch.zeros(rows, (k + 15) // 16 * 16, dtype=torch.int8, device="cuda")
    step = max(1, (1 << 28) // k)
    for at in range(0, rows, step):
        x = torch.randn(min(step, rows - at), k, generator=g, device="cuda")
        store[at:at + step, :k] = torch.round(x * (127 / x.abs().amax(1, keepdim=True))).to(torch.int8)
    return store[:, :k]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.rand(*s, generator=g, device="cuda")        # noqa: E731
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")      # noqa: E731
    st = dict(case=case)
    if case["op"] == "quant":
        m, k = case["m"], case["k"]
        stored = m + 7 if case["gather"] else m
        x = randn(stored, k) * torch.exp2(4 * rand(stored, 1) - 2)       # tokens differ in spread, and have a few
        x *= torch.where(rand(1, k) < 0.003, 12.0, 1.0)                  # channels far above the others
        st["x"] = x.bfloat16() if case["type"] == "bf16" else x
        st["idx"] = torch.randperm(stored, generator=g, device="cuda")[:m].int() if case["gather"] else None
    elif case["op"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        st["a"], st["sa"] = _codes(m, k, g), torch.exp2(rand(m) * 2 - 6)
        st["w"], st["sw"] = _codes(n, k, g), (0.5 + rand(n)) * 0.06 / 127
        if case["mode"] == 3:
            st["w2"], st["sw2"] = _codes(n, k, g), (0.5 + rand(n)) * 0.06 / 127
    else:
        p, v, reqs = _plan(case), case["v"], case["reqs"]
        ints = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()    # noqa: E731
        st["logits"] = randn(p["rows"], v) * 3
        if case["type"] == "bf16":
            st["logits"] = st["logits"].bfloat16()
        st["mask_id"] = v - 1
        st["row_req"] = ints(p["row_req"])
        end = np.cumsum(p["ctx"])
        st["begin"], st["gen"], st["end"] = ints(end - p["ctx"]), ints(end - p["ctx"] + p["gen"]), ints(end)
        # text repeats itself: low ids are frequent; some positions are still masked
        tok = (v * rand(int(end[-1])) ** 3).int().clamp_(0, v - 2)
        st["ctx"] = torch.where(rand(int(end[-1])) < 0.03, v - 1, tok).int()
        st["repetition"] = 1 + 0.5 * rand(reqs)
        st["presence"], st["frequency"] = 0.8 * rand(reqs) - 0.2, 0.4 * rand(reqs)
        st["bias_at"] = ints(np.concatenate([[0], np.cumsum(p["bias"])]))
        r = np.random.RandomState(seed % (1 << 32))
        ids = [np.sort(r.choice(v, b, replace=False)) for b in p["bias"]]
        st["bias_tok"] = ints(np.concatenate(ids + [np.zeros(0)]))
        st["bias_val"] = randn(int(p["bias"].sum())) * 4
        if case["masks"]:
            n, words = case["masks"], (v + 31) // 32
            # a grammar leaves a handful of tokens, a class of them, or nearly all
            keep = torch.tensor([0.0003, 0.1, 0.5, 0.99], device="cuda")[torch.randint(0, 4, (n,), generator=g, device="cuda")]
            weight = 2 ** torch.arange(32, device="cuda")
            bits = torch.empty(n, words, dtype=torch.int32, device="cuda")
            for at in range(0, n, 64):
                some = rand(min(64, n - at), words, 32) < keep[at:at + 64, None, None]
                bits[at:at + 64] = (some * weight).sum(2).to(torch.int32)
            st["allowed"], st["row_mask"] = bits, ints(p["row_mask"])
    return st


# ---- one pass ----------------------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return _own(state)
    return {"quant": _quant, "gemm": _gemm, "rules": _rules, "conf": _conf}[op](state)


def _own(s):
    from paper_2607_08930_b200 import binding as B
    op = s["case"]["op"]
    if op == "quant":
        return B.op_quant_i8(s["x"], idx=s["idx"])
    if op == "gemm":
        return B.op_gemm_i8(s["a"], s["sa"], s["w"], s["sw"], mode=s["case"]["mode"], W2=s.get("w2"), w2_scale=s.get("sw2"))
    if "rules" not in s:            # a program makes it once and updates the tensors that it names
        rep = s["case"]["rep"]
        s["rules"] = B.logit_rules(
            s["case"]["v"], s["row_req"], s["case"]["reqs"], mask_id=s["mask_id"],
            ctx=s["ctx"] if rep else None, ctx_begin=s["begin"] if rep else None, ctx_gen=s["gen"] if rep else None,
            ctx_end=s["end"] if rep else None, repetition=s["repetition"] if rep else None,
            presence=s["presence"] if rep else None, frequency=s["frequency"] if rep else None,
            bias_at=s["bias_at"], bias_tok=s["bias_tok"], bias_val=s["bias_val"],
            allowed=s.get("allowed"), row_mask=s.get("row_mask"))
    if op == "rules":
        if "out" not in s:
            s["out"] = torch.empty_like(s["logits"])
        return B.op_logit_rules(s["logits"], s["rules"], out=s["out"])
    return B.op_rules_confidence(s["logits"], s["rules"])


def _quant(s):
    x = s["x"] if s["idx"] is None else s["x"][s["idx"].long()]
    x = x.float()
    scale = (x.abs().amax(1) / 127).clamp_min(2.0 ** -126)
    codes = torch.round(x.double() / scale.double()[:, None])       # a quotient in 32 bits may land on a half
    return codes.to(torch.int8), scale


def _gemm(s):
    a = s["a"].double()                                              # sums beyond 2^24: exact in 64 bits only
    z = (a @ s["w"].double().T).float() * s["sw"] * s["sa"][:, None]
    if s["case"]["mode"] == 3:
        u = (a @ s["w2"].double().T).float() * s["sw2"] * s["sa"][:, None]
        return (z / (1 + torch.exp(-z)) * u).bfloat16()
    return z if s["case"]["mode"] == 2 else z.bfloat16()


def _ruled(s):
    """The logits after the rules, fp32: repetition, frequency and presence, bias, then what is not allowed at -inf."""
    c = s["case"]
    v, reqs = c["v"], c["reqs"]
    req = s["row_req"].long()
    y = s["logits"].float()
    if c["rep"]:
        t = torch.arange(s["ctx"].numel(), device="cuda")
        owner = torch.searchsorted(s["end"].long(), t, right=True)
        id_ = s["ctx"].long()
        real = (id_ != s["mask_id"]).float()
        seen = torch.zeros(reqs, v, device="cuda").index_put_((owner, id_), real, accumulate=True)
        made = torch.zeros(reqs, v, device="cuda").index_put_((owner, id_), real * (t >= s["gen"].long()[owner]), accumulate=True)
        rho = s["repetition"][req][:, None]
        y = torch.where(seen[req] > 0, torch.where(y > 0, y / rho, y * rho), y)
        less = s["frequency"][:, None] * made + s["presence"][:, None]
        y = torch.where(made[req] > 0, y - less[req], y)
    n = s["bias_tok"].numel()
    owner = torch.searchsorted(s["bias_at"][1:].long(), torch.arange(n, device="cuda"), right=True)
    bias = torch.zeros(reqs, v, device="cuda").index_put_((owner, s["bias_tok"].long()), s["bias_val"], accumulate=True)
    y = y + bias[req]
    if "allowed" in s:
        bit = torch.arange(v, device="cuda")
        keep = (s["allowed"][:, bit // 32] >> (bit % 32).int()) & 1
        some = s["row_mask"].long()
        y = torch.where((some[:, None] >= 0) & (keep[some.clamp_min(0)] == 0), -math.inf, y)
    y[:, s["mask_id"]] = -math.inf
    return y


def _rules(s):
    return _ruled(s).to(s["logits"].dtype)


def _conf(s):
    y = _ruled(s)
    top = y.amax(1, keepdim=True)
    at = torch.arange(y.shape[1], device="cuda", dtype=torch.int32)
    tok = torch.where(y == top, at, y.shape[1]).amin(1)              # the lowest of equal ones
    some = top[:, 0] > -math.inf
    total = torch.exp(y - torch.where(some, top[:, 0], 0.0)[:, None]).sum(1)
    return torch.where(some, tok, -1).int(), torch.where(some, 1 / torch.where(some, total, 1.0), 0.0)


# ---- the same in 64 bits, from the definitions -------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quant":
        x = s["x"].double() if s["idx"] is None else s["x"].double().index_select(0, s["idx"].long())
        scale = (x.abs().max(1).values / 127).float().clamp(min=2.0 ** -126)        # held in fp32
        q = (x / scale.double().unsqueeze(1)).abs()
        low = q.floor()
        up = (q - low > 0.5) | ((q - low == 0.5) & (low % 2 == 1))
        return (torch.sign(x) * (low + up)).to(torch.int8), scale.double()
    if case["op"] == "gemm":
        def product(w, sw):
            x = s["a"].double() * s["sa"].double().unsqueeze(1)
            return torch.cat([torch.mm(x, (b.double() * t.double().unsqueeze(1)).t())
                              for b, t in zip(w.split(8192), sw.split(8192))], 1)
        z = product(s["w"], s["sw"])
        return z * torch.sigmoid(z) * product(s["w2"], s["sw2"]) if case["mode"] == 3 else z
    p, v = _plan(case), case["v"]
    y = s["logits"].double()
    ctx, starts = s["ctx"].cpu().numpy(), s["begin"].cpu().numpy()
    at, tok = s["bias_at"].cpu().numpy(), s["bias_tok"].cpu().numpy()
    first = np.concatenate([[0], np.cumsum(np.bincount(p["row_req"], minlength=case["reqs"]))])
    for i in range(case["reqs"]):
        rows = y[first[i]:first[i + 1]]
        if case["rep"]:
            ids = ctx[starts[i]:starts[i] + p["ctx"][i]]
            every, tail = ids[ids != s["mask_id"]], ids[p["gen"][i]:]
            u = torch.from_numpy(np.unique(every)).long().cuda()
            rho = s["repetition"][i].double()
            rows[:, u] = torch.minimum(rows[:, u] * rho, rows[:, u] / rho)           # rho >= 1: the smaller of the two
            w, count = np.unique(tail[tail != s["mask_id"]], return_counts=True)
            w, count = torch.from_numpy(w).long().cuda(), torch.from_numpy(count).double().cuda()
            rows[:, w] -= s["frequency"][i].double() * count + s["presence"][i].double()
        b = slice(at[i], at[i + 1])
        rows[:, torch.from_numpy(tok[b]).long().cuda()] += s["bias_val"][b].double()
    if case["masks"]:
        for r in range(p["rows"]):
            if p["row_mask"][r] >= 0:
                word = s["allowed"][p["row_mask"][r]].cpu().numpy().view(np.uint8)
                off = np.unpackbits(word, bitorder="little")[:v] == 0
                y[r, torch.from_numpy(off).cuda()] = -math.inf
    y[:, s["mask_id"]] = -math.inf
    if case["op"] == "rules":
        return y
    best, some = y.argmax(1), (y > -math.inf).any(1)
    best = torch.stack([(row == row[b]).nonzero()[0, 0] for row, b in zip(y, best)])
    conf = torch.exp(y.gather(1, best[:, None])[:, 0] - torch.logsumexp(y, 1))
    return torch.where(some, best, -1).int(), torch.where(some, conf, 0.0)
