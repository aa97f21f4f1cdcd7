"""Measurable cases of what a generating step of the decoder runs between its matrix products.

A member of the population that is judged by sampled answers takes a step a token: norms around
each block and the residual sum between them, keys and values written to the cache and attended
over, and the next token drawn from the logits.  The cache holds 8 bits a value where many long
rollouts are to fit.

Case kinds:
  norm     residual sum with the norms before and after a block (copes.residual_norm)
  sample   the next token of a batch of logits from given random numbers (copes.sample_tokens)
  write8   keys and values of tokens into an 8-bit cache and back (copes.cache_append / cache_read)
  attend8  one new token of every sequence over an 8-bit cache (copes.paged_attention)

An 8-bit cache holds the head_dim values of a token's key (or value) of one head as codes, e4m3, and
one exponent e of 127 more: value = code * 2^(e - 127).  A layer's part of a page is
[2][kv_heads][page_size][head_dim] codes, then [2][kv_heads][page_size] exponents, padded to 16 bytes.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
VOCAB = 151936  # of the repository's decoder-shaped workloads


# ------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token of the 0.5B decoder after a block: latency alone
        _norm("norm-one-token", rows=1, hidden=896),
        # heads of the 4B decoder's queries, a batch of prompts: the norm alone, of short rows
        _norm("norm-heads", rows=32 * 700, hidden=128, block=False),
        # prompts through an 8B decoder with norms on both sides of a block, a gate a channel and a residual scale
        _norm("norm-sandwich", rows=16384, hidden=4096, out_norm=True, gate="channel", scale=0.7),
        # fp32 weights, an odd width, a gate of every token's own, rows of a wider buffer
        _norm("norm-fp32-odd", rows=301, hidden=2561, dtype="fp32", out_norm=True, gate="token", strided=True),
        # one rollout's next token, with the usual cuts
        _sample("sample-one", rows=1, top_k=50, top_p=0.95),
        # a decode step of a batch of rollouts, the likeliest tokens that hold 95%
        _sample("sample-step", rows=96, top_p=0.95),
        # a population's rollouts drawn from the whole vocabulary
        _sample("sample-population", rows=2048, scale=1.25),
        # constrained decoding in fp32: a third of an odd vocabulary masked, some rows wholly
        _sample("sample-masked-fp32", rows=301, vocab=32003, min_p=0.02, top_k=200, dtype="fp32", masked=0.35),
        # a decode step of 64 rollouts: one token each
        _write("write8-step", sequences=64, tokens=1, longest=4096),
        # prompts of the 4B decoder read at once
        _write("write8-prompts", sequences=16, tokens=2000, longest=2000),
        # one rollout of the 0.5B decoder shortly after its prompt
        _attend("attend8-one-short", n=1, longest=37, q_heads=14, kv_heads=2, head_dim=64),
        # a population's rollouts with long chains of thought, one slot still empty
        _attend("attend8-large", n=128, longest=16384, layers=2, empty=1),
    ]


def _norm(name, **kw):
    case = {"name": name, "kind": "norm", "rows": 1, "hidden": 896, "dtype": "bf16", "block": True, "out_norm": False,
            "gate": "none", "scale": 1.0, "strided": False}
    return {**case, **kw}


def _sample(name, **kw):
    case = {"name": name, "kind": "sample", "rows": 1, "vocab": VOCAB, "top_k": 0, "top_p": 1.0, "min_p": 0.0, "dtype": "bf16",
            "scale": 1.0, "masked": 0.0}
    return {**case, **kw}


def _write(name, **kw):
    case = {"name": name, "kind": "write8", "sequences": 1, "tokens": 1, "longest": 64, "kv_heads": 8, "head_dim": 128,
            "page_size": 16, "layers": 2, "lens_seed": 5}
    return {**case, **kw}


def _attend(name, **kw):
    case = {"name": name, "kind": "attend8", "n": 1, "longest": 1, "q_heads": 32, "kv_heads": 8, "head_dim": 128,
            "page_size": 16, "layers": 1, "empty": 0, "lens_seed": 5}
    return {**case, **kw}


HEADS = [(14, 2, 64), (32, 8, 128), (16, 16, 64), (24, 3, 128), (15, 5, 80), (16, 1, 128), (12, 4, 256), (40, 8, 96), (6, 2, 16)]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["norm", "sample", "sample", "write8", "attend8"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if kind == "norm":
        hidden = rng.choice([64, 128, 896, 2560, 4096, spread(1, 16384), spread(1, 16384)])
        rows = min(spread(1, 16384), (1 << 25) // hidden)
        block = rng.random() < 0.8
        case = _norm("", rows=rows, hidden=hidden, dtype=dtype, block=block, out_norm=block and rng.random() < 0.5,
                     gate=rng.choice(["none", "channel", "token"]) if block else "none",
                     scale=rng.choice([1.0, 0.7, -0.3]) if block else 1.0, strided=rng.random() < 0.3)
    elif kind == "sample":
        vocab = rng.choice([VOCAB, VOCAB, spread(2, 300000)])
        rows = max(1, min(spread(1, 2048), (1 << 28) // vocab))
        case = _sample("", rows=rows, vocab=vocab, top_k=rng.choice([0, 0, 1, 20, 50, 1000]), top_p=rng.choice([1.0, 0.9, 0.95, 0.5]),
                       min_p=rng.choice([0.0, 0.0, 0.05]), dtype=dtype, scale=rng.choice([1.0, 1.0, 0.7, 1.43]),
                       masked=rng.choice([0.0, 0.0, 0.4]))
    else:
        q, kv, d = rng.choice(HEADS)
        page = rng.choice([16, 16, 32, 64, 8, 7, 50])
        if kind == "write8":
            sequences, tokens = spread(1, 64), rng.choice([1, 1, spread(1, 2000)])
            while sequences * tokens * kv * d > 1 << 25:
                tokens = max(1, tokens // 2)
            case = _write("", sequences=sequences, tokens=tokens, longest=max(tokens, spread(1, 2000)), kv_heads=kv, head_dim=d,
                          page_size=page, layers=rng.choice([1, 2, 3]))
        else:
            n, longest = spread(1, 128), spread(1, 131071)
            longest = max(1, min(longest, (2 << 30) // (n * kv * d * 2)))
            case = _attend("", n=n, longest=longest, q_heads=q, kv_heads=kv, head_dim=d, page_size=page,
                           layers=rng.choice([1, 2, 3]), empty=rng.choice([0, 0, 1]) if n > 1 else 0)
        case["lens_seed"] = rng.randrange(1 << 30)
    del case["name"]
    return case


# ------------------------------------------------------------- sizes that the cases imply
def _lengths(case):
    """Lengths of the case's sequences (host); the first is the longest."""
    rng = np.random.default_rng(case["lens_seed"])
    n = case["n"] if case["kind"] == "attend8" else case["sequences"]
    lens = rng.integers(case.get("tokens", 1), case["longest"] + 1, n)
    lens[0] = case["longest"]
    if case.get("empty"):
        lens[n - case["empty"]:] = 0
    return lens


def _layer_bytes(case):
    heads = 2 * case["kv_heads"] * case["page_size"]
    return -(-heads * (case["head_dim"] + 1) // 16) * 16


def _size(case):
    return 2 if case["dtype"] == "bf16" else 4


def work(case):
    if case["kind"] == "norm":
        cells, size = case["rows"] * case["hidden"], _size(case)
        arrays = 2  # x in, its norm out
        if case["block"]:
            arrays += 2 + (case["gate"] == "token")  # the block's output, the sum, a gate of every token's own
        vectors = 1 + case["out_norm"] + (case["gate"] == "channel")
        return {"bytes": (arrays * cells + vectors * case["hidden"]) * size, "flops": 4 * cells * (1 + case["block"])}
    if case["kind"] == "sample":
        cells = case["rows"] * case["vocab"]
        return {"bytes": cells * _size(case) + 20 * case["rows"], "flops": 16 * cells}
    heads, d = 2 * case["kv_heads"], case["head_dim"]
    if case["kind"] == "write8":
        rows = case["sequences"] * case["tokens"]
        return {"bytes": rows * (heads * 2 * (2 * d + d + 1) + 8), "flops": 4 * rows * heads * d}
    tokens, rows = int(_lengths(case).sum()), case["n"] * case["q_heads"]
    pages = int((-(-_lengths(case) // case["page_size"])).sum())
    io = rows * (2 * d * 2 + 4) + 4 * (pages + 2 * case["n"])
    return {"bytes": tokens * heads * (d + 1) + io, "flops": 4 * tokens * case["q_heads"] * d}


# ------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)

    def normal(*shape, dtype=torch.bfloat16, scale=1.0, mean=0.0):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dtype).mul_(scale).add_(mean)

    if case["kind"] == "norm":
        rows, hidden, dtype = case["rows"], case["hidden"], DTYPES[case["dtype"]]

        def matrix(scale, mean=0.0):
            wide = normal(rows, hidden + (24 if case["strided"] else 0), dtype=dtype, scale=scale, mean=mean)
            return wide[:, :hidden]

        s.update(x=matrix(3.0), weight=normal(hidden, dtype=dtype, scale=0.1, mean=1.0), y=None, out_weight=None, gate_by=None)
        if case["block"]:
            s["y"] = matrix(1.5)
            if case["out_norm"]:
                s["out_weight"] = normal(hidden, dtype=dtype, scale=0.1, mean=1.0)
            if case["gate"] == "channel":
                s["gate_by"] = normal(hidden, dtype=dtype, scale=0.2, mean=0.5)
            elif case["gate"] == "token":
                s["gate_by"] = matrix(0.2, 0.5)
        return s

    if case["kind"] == "sample":
        rows, vocab, dtype = case["rows"], case["vocab"], DTYPES[case["dtype"]]
        # most tokens are far off; a few stand out, in some rows more than in others
        logits = normal(rows, vocab, dtype=dtype, scale=1.5)
        few = min(64, vocab)
        first = torch.randint(0, vocab, (rows, 1), generator=gen, device="cuda")
        ids = (first + torch.arange(few, device="cuda") * (vocab // few)) % vocab
        sure = 0.6 + 0.6 * torch.rand(rows, 1, generator=gen, device="cuda")
        high = sure * (18.0 - 2.5 * torch.log(torch.arange(1, few + 1, device="cuda")))
        logits.scatter_(1, ids, high.to(dtype))
        if case["masked"]:
            for a in range(0, rows, 512):
                part = logits[a:a + 512]
                part.masked_fill_(torch.rand(part.shape, generator=gen, device="cuda") < case["masked"], -math.inf)
            logits[::97] = -math.inf  # no token allowed
        s.update(logits=logits, u=torch.rand(rows, generator=gen, device="cuda"))
        return s

    lens, ps, kv, d = _lengths(case), case["page_size"], case["kv_heads"], case["head_dim"]
    pages = -(-lens // ps)
    total = int(pages.sum())
    n_pages = total + total // 8 + 1
    ids = np.random.default_rng(case["lens_seed"] + 1).permutation(n_pages)[:total].astype(np.int32)
    table = np.full((len(lens), int(pages.max())), -1, np.int32)
    at = 0
    for i, p in enumerate(pages):
        table[i, :p] = ids[at:at + p]
        at += p
    refs = np.zeros(n_pages, np.int32)
    refs[ids] = 1
    pool = torch.zeros(n_pages, case["layers"], _layer_bytes(case), dtype=torch.uint8, device="cuda")
    codes = 2 * kv * ps * d
    if case["kind"] == "attend8":
        # values of a standard deviation of 1 or a few, in codes of up to 448
        pool[..., :codes] = normal(n_pages, case["layers"], codes, scale=120.0).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        pool[..., codes:codes + 2 * kv * ps] = torch.randint(118, 122, (n_pages, case["layers"], 2 * kv * ps), generator=gen, device="cuda",
                                                             dtype=torch.uint8)
        qkv = normal(case["n"], (case["q_heads"] + 2 * kv) * d, scale=1.5)  # q rows are a slice of the fused projection's output
        s.update(q=qkv[:, :case["q_heads"] * d].unflatten(1, (case["q_heads"], d)), softmax_scale=d ** -0.5)
    else:
        rows = len(lens) * case["tokens"]
        qkv = normal(rows, 3 * kv * d, scale=1.5)
        qkv[:, ::37] *= 20.0  # channels that stand out
        last = np.arange(case["tokens"]) - case["tokens"]
        s.update(k=qkv[:, kv * d:2 * kv * d].unflatten(1, (kv, d)), v=qkv[:, 2 * kv * d:].unflatten(1, (kv, d)),
                 slots=torch.arange(len(lens), dtype=torch.int32, device="cuda").repeat_interleave(case["tokens"]),
                 position=torch.from_numpy((lens[:, None] + last).astype(np.int32).ravel()).cuda())
    s.update(pool=pool, table=torch.from_numpy(table).cuda(), length=torch.from_numpy(lens.astype(np.int32)).cuda(),
             refs=torch.from_numpy(refs).cuda(), layer=case["layers"] - 1)
    if own:
        from paper_2608_02391_gb300 import copes
        s["cache"] = copes.KVCache(s["pool"], s["table"], s["length"], s["refs"], heads=(kv, ps, d))
    return s


# --------------------------------------------------------------------------------- runs
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2608_02391_gb300 import copes
    if s["kind"] == "norm":
        total, normed = copes.residual_norm(s["x"], s["weight"], y=s["y"], out_weight=s["out_weight"], gate=s["gate_by"],
                                            scale=s["scale"], eps=1e-6)
        return [normed] if s["y"] is None else [total, normed]
    if s["kind"] == "sample":
        r = copes.sample_tokens(s["logits"], s["u"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], scale=s["scale"])
        return [r.ids, r.logprob, r.kept]
    if s["kind"] == "write8":
        copes.cache_append(s["cache"], s["layer"], s["k"], s["v"], slots=s["slots"], position=s["position"])
        k, v = copes.cache_read(s["cache"], s["layer"], slots=s["slots"], position=s["position"])
        return [k, v]
    out, lse = copes.paged_attention(s["cache"], s["layer"], s["q"], scale=s["softmax_scale"])
    return [out, lse]


def _run_plain(s):
    return {"norm": _plain_norm, "sample": _plain_sample, "write8": _plain_write, "attend8": _plain_attend}[s["kind"]](s)


def _plain_norm(s):
    dtype, x = s["x"].dtype, s["x"].float()
    total = x
    if s["y"] is not None:
        z = s["y"].float()
        if s["out_weight"] is not None:
            z = z * torch.rsqrt((z * z).mean(1, keepdim=True) + 1e-6) * s["out_weight"].float()
        if s["gate_by"] is not None:
            z = z * s["gate_by"].float()
        total = x + z * s["scale"]
    normed = total * torch.rsqrt((total * total).mean(1, keepdim=True) + 1e-6) * s["weight"].float()
    return [normed.to(dtype)] if s["y"] is None else [total.to(dtype), normed.to(dtype)]


# The weight of a token whose logit is the largest's less d is, with t = d * scale * log2(e) in fp32, n = floor(t) and
# f = t - n, the whole number floor(P(f) 2^(40 - n)), P(f) within 2^-21 of 2^-f: a polynomial whose every step is rounded
# to fp32.  Sums of whole numbers are the same in any order, and so is the token that they lead to.
_P = [1.0, -0.693140983581543, 0.2401522845029831, -0.05521015450358391, 0.009098555892705917, -0.0008996404358185828]


def _fused(p, f, c):
    """p f + c, rounded once: the product is exact in 64 bits."""
    return (p.double() * f.double() + c).float()


def _distance(x, top, scale):
    return ((top - x) * float(np.float32(scale) * np.float32(1.44269504088896340736))).clamp(max=63.0)


def _plain_sample(s):
    x, u = s["logits"].float() + 0.0, s["u"]
    top = x.amax(1, keepdim=True).clamp(min=-3.4028234663852886e38)
    t = _distance(x, top, s["scale"])
    n = torch.floor(t)
    f = t - n
    p = _fused(_fused(_fused(_fused(_fused(torch.full_like(f, _P[5]), f, _P[4]), f, _P[3]), f, _P[2]), f, _P[1]), f, _P[0])
    weight = ((p * 2.0 ** 24).long() << 16) >> n.long()
    weight = weight.masked_fill(x == -math.inf, 0)
    kept = weight > 0
    if s["min_p"] > 0:
        kept = kept & (t <= float(np.float32(-math.log2(float(np.float32(s["min_p"]))))))
    if s["top_k"] or s["top_p"] < 1:
        ids = torch.sort(x, dim=1, descending=True, stable=True)[1]
        ordered = weight.gather(1, ids)
        before = torch.ones_like(ordered, dtype=torch.bool)
        if s["top_k"]:
            before[:, s["top_k"]:] = False
            ordered = ordered.masked_fill(~before, 0)
        if s["top_p"] < 1:
            total = ordered.sum(1, keepdim=True).double()
            need = torch.ceil(total * float(np.float32(s["top_p"]))).long()
            before = before & (torch.cumsum(ordered, 1) - ordered < need)
        kept = kept & torch.zeros_like(kept).scatter_(1, ids, before)
    sums = torch.cumsum(weight.masked_fill(~kept, 0), 1)
    total = sums[:, -1]
    r = torch.floor(u.double() * 2.0 ** 31).long()
    place = (total >> 31) * r + (((total & ((1 << 31) - 1)) * r) >> 31)
    drawn = (sums <= place[:, None]).sum(1)
    none = total == 0
    far = t.gather(1, drawn.clamp(max=x.shape[1] - 1)[:, None])[:, 0].double()
    logprob = -(far * math.log(2.0) + torch.log1p((total - (1 << 40)).double() * 2.0 ** -40)).float()
    return [drawn.masked_fill(none, -1), (logprob + 0.0).masked_fill(none, math.nan), kept.sum(1).to(torch.int32)]


def _parts(s):
    """Codes [pages, 2, kv, ps, d] and exponents [pages, 2, kv, ps] of the layer, views of the pool."""
    kv, ps, d = s["kv_heads"], s["page_size"], s["head_dim"]
    layer = s["pool"][:, s["layer"]]
    codes = 2 * kv * ps * d
    return layer[:, :codes].unflatten(1, (2, kv, ps, d)), layer[:, codes:codes + 2 * kv * ps].unflatten(1, (2, kv, ps))


def _values(codes, exponents):
    return codes.contiguous().view(torch.float8_e4m3fn).float() * torch.exp2(exponents.float() - 127.0)[..., None]


def _plain_write(s):
    codes, exponents = _parts(s)
    page = s["table"][s["slots"].long(), (s["position"] // s["page_size"]).long()].long()
    place = (s["position"] % s["page_size"]).long()
    x = torch.stack((s["k"], s["v"]), 1).float()
    # the power of two that brings a row's largest finite value into (224, 448]
    most = x.abs().masked_fill(~torch.isfinite(x), 0.0).amax(3).double()
    mantissa, power = torch.frexp(most)
    e = torch.where(most > 0, power - 9 + (mantissa > 0.875), -126).clamp(min=-126)
    scaled = (x.double() * torch.exp2(-e.double())[..., None]).float()
    exponents[page, :, :, place] = (e + 127).to(torch.uint8)
    codes[page, :, :, place] = scaled.to(torch.float8_e4m3fn).view(torch.uint8)
    read = _values(codes[page, :, :, place], exponents[page, :, :, place]).to(torch.bfloat16)
    return [read[:, 0], read[:, 1]]


def _plain_attend(s):
    q, length, kv = s["q"].float(), s["length"], s["kv_heads"]
    n, hq, d = q.shape
    codes, exponents = _parts(s)
    table = s["table"].clamp(min=0).long()
    pages = _values(codes[table], exponents[table])  # [n, width, 2, kv, ps, d]
    keys, values = pages[:, :, 0].transpose(1, 2).flatten(2, 3), pages[:, :, 1].transpose(1, 2).flatten(2, 3)
    scores = torch.matmul(q.view(n, kv, hq // kv, d), keys.transpose(2, 3)) * s["softmax_scale"]
    there = torch.arange(scores.shape[3], device="cuda") < length[:, None]
    scores = scores.masked_fill(~there[:, None, None], -math.inf)
    top = scores.amax(3, keepdim=True)
    p = torch.exp(scores - top.clamp(min=-3e38))
    total = p.sum(3, keepdim=True)
    values = values.masked_fill(~there[:, None, :, None], 0.0)
    out = torch.matmul(p, values) / total.clamp(min=1e-38)
    lse = (top + torch.log(total)).view(n, hq)
    return [out.view(n, hq, d).to(s["q"].dtype), lse]


# ------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        return _exact_norm(s)
    if case["kind"] == "sample":
        at_once = max(1, (1 << 23) // case["vocab"])
        return [None, torch.cat([_exact_sample(s, a, a + at_once) for a in range(0, case["rows"], at_once)]), None]
    if case["kind"] == "write8":
        return [_exact_stored(s["k"].double()), _exact_stored(s["v"].double())]
    return _exact_attend(s, case)


def _exact_norm(s):
    def unit(a):
        return a / torch.sqrt(a.square().sum(1, keepdim=True) / a.shape[1] + 1e-6)

    x = s["x"].double()
    if s["y"] is None:
        return [unit(x) * s["weight"].double()]
    z = s["y"].double()
    if s["out_weight"] is not None:
        z = unit(z) * s["out_weight"].double()
    if s["gate_by"] is not None:
        z = s["gate_by"].double() * z
    x = x + s["scale"] * z
    return [x, unit(x) * s["weight"].double()]


def _exact_sample(s, a, b):
    """Log probabilities of the tokens of rows [a, b): which ones these are by the weights' definition, the rest in 64 bits."""
    x, order = torch.sort(-s["logits"][a:b].double(), dim=1, stable=True)
    none = torch.isposinf(x[:, :1])
    x = -x
    factor = float(np.float32(s["scale"]) * np.float32(1.44269504088896340736))
    t = ((x[:, :1] - x).float().double() * factor).float().double().nan_to_num(nan=1e4, posinf=1e4)
    f = t % 1.0
    p = torch.zeros_like(f)
    for c in reversed(_P):
        p = (p * f + c).float().double()
    w = torch.floor(torch.ldexp(p, 40 - (t - f).clamp(max=1000))).long()
    rank = torch.arange(w.shape[1], device="cuda")
    if s["top_k"]:
        w = torch.where(rank < s["top_k"], w, 0)
    if s["top_p"] < 1:
        need = torch.ceil(w.sum(1).double() * float(np.float32(s["top_p"])))
        w = torch.where(rank <= (torch.cumsum(w, 1) < need[:, None]).sum(1, keepdim=True), w, 0)
    if s["min_p"] > 0:
        w = torch.where(t > float(np.float32(-math.log2(float(np.float32(s["min_p"]))))), 0, w)
    sums = torch.cumsum(torch.zeros_like(w).scatter_(1, order, w), 1)
    place = [int(u * 2.0 ** 31) * total >> 31 for u, total in zip(s["u"][a:b].tolist(), sums[:, -1].tolist())]
    drawn = (sums <= torch.tensor(place, device="cuda")[:, None]).sum(1, keepdim=True)
    logp = torch.log_softmax(torch.where(w > 0, x * s["scale"], -math.inf), 1)
    return torch.where(none, math.nan, logp.masked_fill(order != drawn, 0.0).nan_to_num(nan=0.0).sum(1, keepdim=True))[:, 0]


def _exact_stored(x):
    """What 8 bits hold of rows x: 4 significant bits, less below 2^-6 of codes of up to 448."""
    most = x.abs().amax(2, keepdim=True).clamp(min=2.0 ** -126)
    mantissa, power = torch.frexp(most / 448.0)
    unit = torch.exp2(torch.where(mantissa == 0.5, power - 1, power).double())
    code = x / unit
    step = torch.exp2(torch.floor(torch.log2(code.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(code / step) * step * unit


def _exact_attend(s, case):
    n, hq, d = s["q"].shape
    kv, ps = case["kv_heads"], case["page_size"]
    out = torch.zeros(n, hq, d, dtype=torch.float64, device="cuda")
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64, device="cuda")
    sign, power, low = (torch.arange(256, device="cuda") >> 7), (torch.arange(256, device="cuda") >> 3) & 15, torch.arange(256, device="cuda") & 7
    magnitude = torch.where(power > 0, torch.ldexp(1.0 + low.double() / 8, power - 7), low.double() * 2.0 ** -9)
    held = torch.where(sign > 0, -magnitude, magnitude)
    for i, count in enumerate(_lengths(case).tolist()):
        if not count:
            continue
        layer = s["pool"][s["table"][i, :-(-count // ps)].long(), s["layer"]]
        code = layer[:, :2 * kv * ps * d].reshape(-1, 2, kv, ps, d)
        power_of = layer[:, 2 * kv * ps * d:2 * kv * ps * (d + 1)].reshape(-1, 2, kv, ps).double()
        for g in range(kv):
            both = held[code[:, :, g].long()] * torch.exp2(power_of[:, :, g] - 127)[..., None]
            keys, values = both[:, 0].reshape(-1, d)[:count], both[:, 1].reshape(-1, d)[:count]
            rows = slice(g * (hq // kv), (g + 1) * (hq // kv))
            z = s["q"][i, rows].double() @ keys.T * s["softmax_scale"]
            lse[i, rows] = torch.logsumexp(z, 1)
            out[i, rows] = torch.softmax(z, 1) @ values
    return [out, lse]
