"""Measurable cases of the operators that answer with the weights under evolution.

A member of the population is judged by what its perturbed weights answer: its rollouts attend
over a paged key-value cache one token at a time, the rollouts of one prompt share the prompt's
pages, and a scored answer's reward is read off the log probabilities of its tokens.

Case kinds:
  attend    one new token of every sequence over its pages (copes.paged_attention)
  fork      rollouts of shared prompts begin and end: fork, grow by a token, append its key and
            value in one layer, free (copes.cache_fork / _grow / _append / _free)
  compact   the pages in use of a sparse pool moved together (copes.cache_compact)
  logprobs  log probabilities, entropy and top alternatives of a batch of logits
            (copes.token_logprobs)
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
        # one rollout of the 0.5B decoder shortly after its prompt: latency alone
        _attend("attend-one-short", n=1, longest=37, q_heads=14, kv_heads=2, head_dim=64),
        # the 4B decoder answering a batch of prompts of mixed lengths, one slot still empty
        _attend("attend-batch", n=32, longest=4096, q_heads=32, kv_heads=8, head_dim=128, empty=1),
        # a full population's rollouts with long chains of thought
        _attend("attend-large", n=128, longest=16384, q_heads=32, kv_heads=8, head_dim=128, layers=2),
        # one agentic transcript that fills its context, odd length
        _attend("attend-one-long", n=1, longest=131071, q_heads=32, kv_heads=8, head_dim=128),
        # fp32 weights and cache, pages and heads of unusual sizes
        _attend("attend-fp32-odd", n=7, longest=3001, q_heads=15, kv_heads=5, head_dim=80, page_size=7, dtype="fp32"),
        # the 0.5B decoder: one short prompt answered eight times
        _fork("fork-one-prompt", prompts=1, rollouts=8, longest=37, layers=24, kv_heads=2, head_dim=64),
        # the 4B decoder: 16 prompts answered 16 times each
        _fork("fork-population", prompts=16, rollouts=16, longest=700, layers=36, kv_heads=8, head_dim=128),
        # the 4B decoder's pool after half of the rollouts have ended
        _compact("compact-sparse", n_pages=1500, sequences=64, used=0.5, layers=36, kv_heads=8, head_dim=128),
        # one generated token with its alternatives
        _logprobs("logprobs-one", rows=1, vocab=VOCAB, top=20),
        # one decode step of a batch of rollouts
        _logprobs("logprobs-step", rows=96, vocab=VOCAB, top=5),
        # scored answers: every token of a batch
        _logprobs("logprobs-answers", rows=4096, vocab=VOCAB, top=20),
        # constrained decoding in fp32 at a temperature: a third of an odd vocabulary masked, some
        # rows wholly
        _logprobs("logprobs-masked-fp32", rows=301, vocab=32003, top=8, dtype="fp32", scale=1.25, masked=0.35),
    ]


def _attend(name, **kw):
    case = {"name": name, "kind": "attend", "n": 1, "longest": 1, "q_heads": 14, "kv_heads": 2, "head_dim": 64,
            "page_size": 16, "dtype": "bf16", "layers": 1, "empty": 0, "lens_seed": 5}
    return {**case, **kw}


def _fork(name, **kw):
    case = {"name": name, "kind": "fork", "prompts": 1, "rollouts": 1, "longest": 37, "layers": 1, "kv_heads": 2,
            "head_dim": 64, "page_size": 16, "dtype": "bf16", "lens_seed": 5}
    return {**case, **kw}


def _compact(name, **kw):
    case = {"name": name, "kind": "compact", "n_pages": 64, "sequences": 4, "used": 0.5, "layers": 1, "kv_heads": 2,
            "head_dim": 64, "page_size": 16, "dtype": "bf16", "lens_seed": 5}
    return {**case, **kw}


def _logprobs(name, **kw):
    case = {"name": name, "kind": "logprobs", "rows": 1, "vocab": VOCAB, "top": 0, "dtype": "bf16", "scale": 1.0,
            "masked": 0.0}
    return {**case, **kw}


HEADS = [(14, 2, 64), (32, 8, 128), (16, 16, 64), (24, 3, 128), (15, 5, 80), (16, 1, 128), (12, 4, 256), (40, 8, 96)]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["attend", "attend", "fork", "compact", "logprobs", "logprobs"])
    q, kv, d = rng.choice(HEADS)
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    page = rng.choice([16, 16, 32, 64, 8, 7, 50])
    size = 2 if dtype == "bf16" else 4
    if kind == "attend":
        n, longest = spread(1, 128), spread(1, 131071)
        most = 4 << 30  # bytes of keys and values that the longest rows may hold
        longest = max(1, min(longest, most // (n * kv * d * 2 * size)))
        case = _attend("", n=n, longest=longest, q_heads=q, kv_heads=kv, head_dim=d, page_size=page, dtype=dtype,
                       layers=rng.choice([1, 2, 3]), empty=rng.choice([0, 0, 1]) if n > 1 else 0)
    elif kind == "fork":
        prompts, rollouts, longest, layers = spread(1, 16), spread(1, 16), spread(1, 700), spread(1, 36)
        case = _fork("", prompts=prompts, rollouts=rollouts, longest=longest, layers=layers, kv_heads=kv, head_dim=d,
                     page_size=page, dtype=dtype)
        while _pool_bytes(case) > 3 << 30:
            case["layers"] = max(1, case["layers"] // 2)
            case["longest"] = max(1, case["longest"] // 2)
            case["prompts"] = max(1, case["prompts"] // 2)
    elif kind == "compact":
        case = _compact("", n_pages=spread(16, 1500), sequences=spread(1, 64), used=round(rng.uniform(0.1, 0.95), 3),
                        layers=spread(1, 36), kv_heads=kv, head_dim=d, page_size=page, dtype=dtype)
        while _pool_bytes(case) > 3 << 30:
            case["layers"] = max(1, case["layers"] // 2)
            case["n_pages"] = max(16, case["n_pages"] * 3 // 4)
    else:
        vocab = rng.choice([VOCAB, VOCAB, spread(2, 300000)])
        rows = max(1, min(spread(1, 4096), (1 << 30) // (vocab * size)))
        case = _logprobs("", rows=rows, vocab=vocab, top=min(rng.choice([0, 1, 5, 20, 32]), vocab), dtype=dtype,
                         scale=rng.choice([1.0, 1.0, 0.7, 1.43]), masked=rng.choice([0.0, 0.0, 0.4]))
    if "lens_seed" in case:
        case["lens_seed"] = rng.randrange(1 << 30)
    del case["name"]
    return case


# ------------------------------------------------------------- sizes that the cases imply
def _lengths(case):
    """Lengths of the case's sequences (host); the first is the longest."""
    rng = np.random.default_rng(case["lens_seed"])
    n = case["n"] if case["kind"] == "attend" else case["prompts"]
    lens = rng.integers(1, case["longest"] + 1, n)
    lens[0] = case["longest"]
    if case.get("empty"):
        lens[n - case["empty"]:] = 0
    return lens


def _pages_of(case):
    """Pages in use by each sequence (host)."""
    if case["kind"] != "compact":
        return -(-_lengths(case) // case["page_size"])
    total = max(1, int(case["n_pages"] * case["used"]))
    each = np.full(case["sequences"], total // case["sequences"])
    each[:total % case["sequences"]] += 1
    return each


def _n_pages(case):
    if case["kind"] == "compact":
        return case["n_pages"]
    pages = int(_pages_of(case).sum())
    if case["kind"] == "fork":  # a copied last page and a page to grow into for every rollout
        return pages + 2 * case["prompts"] * case["rollouts"]
    return pages + pages // 8 + 1


def _size(case):
    return 2 if case["dtype"] == "bf16" else 4


def _page_bytes(case):
    return case["layers"] * 2 * case["kv_heads"] * case["page_size"] * case["head_dim"] * _size(case)


def _pool_bytes(case):
    return _n_pages(case) * _page_bytes(case)


def work(case):
    if case["kind"] == "attend":
        lens, rows = _lengths(case), case["n"] * case["q_heads"]
        kv = int(lens.sum()) * case["kv_heads"] * case["head_dim"] * 2 * _size(case)
        io = rows * (2 * case["head_dim"] * _size(case) + 4) + 4 * (int(_pages_of(case).sum()) + 2 * case["n"])
        return {"bytes": kv + io, "flops": 4 * int(lens.sum()) * case["q_heads"] * case["head_dim"]}
    if case["kind"] == "fork":
        lens, ps, r = _lengths(case), case["page_size"], case["rollouts"]
        partly = int((lens % ps != 0).sum())  # read once, written by each of its rollouts
        pages = _pages_of(case)
        tables = 4 * int(pages.sum()) * (1 + 2 * r) + 4 * 2 * int(pages.sum())
        token = 2 * case["kv_heads"] * case["head_dim"] * _size(case)
        return {"bytes": partly * (1 + r) * _page_bytes(case) + tables + 2 * len(lens) * r * token, "flops": 0}
    if case["kind"] == "compact":
        moved = _moved(case)
        return {"bytes": 2 * moved * _page_bytes(case) + 8 * (case["n_pages"] + int(_pages_of(case).sum())), "flops": 0}
    cells = case["rows"] * case["vocab"]
    return {"bytes": cells * _size(case) + case["rows"] * (16 + 12 * case["top"]), "flops": 5 * cells}


def _page_order(case):
    """The ids that the sequences' pages have, in order of sequence and position (host)."""
    rng = np.random.default_rng(case["lens_seed"] + 1)
    return rng.permutation(_n_pages(case))[:int(_pages_of(case).sum())].astype(np.int32)


def _moved(case):
    ids = _page_order(case)
    return int((ids >= len(ids)).sum())


# ------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dtype).mul_(scale)

    s = dict(case)
    if case["kind"] == "logprobs":
        rows, vocab = case["rows"], case["vocab"]
        logits = normal(rows, vocab, scale=2.5)
        targets = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
        if case["masked"]:
            for a in range(0, rows, 512):
                part = logits[a:a + 512]
                part.masked_fill_(torch.rand(part.shape, generator=gen, device="cuda") < case["masked"], -math.inf)
            logits[::97] = -math.inf  # no token allowed
            targets[5::31] = -1       # padding
        logits.scatter_(1, targets.clamp(min=0)[:, None], 9.0)  # a model knows the next token more often than not
        if case["masked"]:
            logits[::97] = -math.inf
        s.update(logits=logits, targets=targets)
        return s

    pages, ids = _pages_of(case), _page_order(case)
    kv, ps, d = case["kv_heads"], case["page_size"], case["head_dim"]
    rollouts = case.get("prompts", 0) * case.get("rollouts", 0)
    width = int(pages.max()) + (1 if case["kind"] == "fork" else 0)
    table = np.full((len(pages) + rollouts, width), -1, np.int32)
    at = 0
    for i, p in enumerate(pages):
        table[i, :p] = ids[at:at + p]
        at += p
    if case["kind"] == "compact":
        last = np.random.default_rng(case["lens_seed"] + 2).integers(1, ps + 1, len(pages))
        lens = np.where(pages > 0, (pages - 1) * ps + last, 0)
    else:
        lens = _lengths(case)
    length = np.concatenate([lens, np.zeros(rollouts, np.int64)]).astype(np.int32)
    refs = np.zeros(_n_pages(case), np.int32)
    refs[ids] = 1
    s.update(pool=normal(_n_pages(case), case["layers"], 2, kv, ps, d), table=torch.from_numpy(table).cuda(),
             length=torch.from_numpy(length).cuda(), refs=torch.from_numpy(refs).cuda())
    if case["kind"] == "attend":
        # q rows are a slice of the fused projection's output
        qkv = normal(case["n"], (case["q_heads"] + 2 * kv) * d, scale=1.5)
        s.update(q=qkv[:, :case["q_heads"] * d].unflatten(1, (case["q_heads"], d)), layer=case["layers"] - 1,
                 scale=d ** -0.5)
    elif case["kind"] == "fork":
        qkv = normal(rollouts, 3 * kv * d)
        s.update(k=qkv[:, kv * d:2 * kv * d].unflatten(1, (kv, d)), v=qkv[:, 2 * kv * d:].unflatten(1, (kv, d)),
                 parents=torch.arange(case["prompts"], dtype=torch.int32, device="cuda").repeat_interleave(case["rollouts"]),
                 children=torch.arange(rollouts, dtype=torch.int32, device="cuda") + case["prompts"],
                 layer=case["layers"] - 1)
    else:
        s.update(table0=s["table"].clone(), refs0=s["refs"].clone())
    if own:
        from paper_2608_02391_gb300 import copes
        s["cache"] = copes.KVCache(s["pool"], s["table"], s["length"], s["refs"])
    return s


# --------------------------------------------------------------------------------- runs
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2608_02391_gb300 import copes
    if s["kind"] == "logprobs":
        r = copes.token_logprobs(s["logits"], s["targets"], top=s["top"], scale=s["scale"])
        return [r.logprob, r.entropy, r.top_ids, r.top_logprobs]
    cache = s["cache"]
    if s["kind"] == "attend":
        out, lse = copes.paged_attention(cache, s["layer"], s["q"], scale=s["scale"])
        return [out, lse]
    if s["kind"] == "fork":
        copes.cache_fork(cache, s["parents"], s["children"])
        copes.cache_grow(cache, s["children"], 1)
        copes.cache_append(cache, s["layer"], s["k"], s["v"], slots=s["children"])
        grown = [s["table"].clone(), s["length"].clone(), s["refs"].clone()]
        copes.cache_free(cache, s["children"])
        return grown + [s["table"], s["length"], s["refs"], s["pool"]]
    s["table"].copy_(s["table0"])  # a sparse pool again: moved pages still hold what they held
    s["refs"].copy_(s["refs0"])
    copes.cache_compact(cache)
    return [s["table"], s["refs"], s["pool"]]


def _run_plain(s):
    return {"attend": _plain_attend, "fork": _plain_fork, "compact": _plain_compact, "logprobs": _plain_logprobs}[s["kind"]](s)


def _plain_attend(s):
    q, length = s["q"].float(), s["length"]
    n, hq, d = q.shape
    kv = s["kv_heads"]
    pages = s["pool"][:, s["layer"]][s["table"].clamp(min=0).long()].float()  # [n, width, 2, kv, ps, d]
    keys, values = pages[:, :, 0].transpose(1, 2).flatten(2, 3), pages[:, :, 1].transpose(1, 2).flatten(2, 3)
    scores = torch.matmul(q.view(n, kv, hq // kv, d), keys.transpose(2, 3)) * s["scale"]
    there = torch.arange(scores.shape[3], device="cuda") < length[:, None]
    scores = scores.masked_fill(~there[:, None, None], -math.inf)
    top = scores.amax(3, keepdim=True)
    p = torch.exp(scores - top.clamp(min=-3e38))
    total = p.sum(3, keepdim=True)
    values = values.masked_fill(~there[:, None, :, None], 0.0)
    out = torch.matmul(p, values) / total.clamp(min=1e-38)
    lse = (top + torch.log(total)).view(n, hq)
    return [out.view(n, hq, d).to(s["q"].dtype), lse]


def _first_free(refs, count):
    """The lowest `count` free pages, ascending."""
    return torch.sort((refs != 0).to(torch.int32), stable=True)[1][:count]


def _plain_fork(s):
    table, length, refs, pool, ps = s["table"], s["length"], s["refs"], s["pool"], s["page_size"]
    parents, children = s["parents"].long(), s["children"].long()
    place = torch.arange(table.shape[1], device="cuda")
    # fork: full pages shared, a partly filled last page copied to the next free page
    lens = length[parents]
    rows, full, partly = table[parents], lens // ps, lens % ps != 0
    shared = place < full[:, None]
    refs.index_add_(0, rows.clamp(min=0).flatten().long(), shared.flatten().to(torch.int32))
    free = _first_free(refs, len(children))
    new = free[(torch.cumsum(partly, 0) - 1).clamp(min=0)]
    last = rows.gather(1, full[:, None].clamp(max=table.shape[1] - 1).long())[:, 0].clamp(min=0).long()
    at, to = last[partly], new[partly]
    pool[to] = pool[at]
    refs[to] = 1
    rows = torch.where(shared, rows, -1)
    table[children] = torch.where(partly[:, None] & (place == full[:, None]), new[:, None].to(torch.int32), rows)
    length[children] = lens
    # grow by one token: a new page where the last one is full
    need = lens % ps == 0
    free = _first_free(refs, len(children))
    new = free[(torch.cumsum(need, 0) - 1).clamp(min=0)]
    rows = table[children]
    table[children] = torch.where(need[:, None] & (place == full[:, None]), new[:, None].to(torch.int32), rows)
    refs[new[need]] = 1
    length[children] = lens + 1
    # append the token's key and value in one layer
    page = table[children, full.long()].long()
    inside = (lens % ps).long()
    pool[page, s["layer"], 0, :, inside] = s["k"]
    pool[page, s["layer"], 1, :, inside] = s["v"]
    grown = [table.clone(), length.clone(), refs.clone()]
    # free
    rows = table[children]
    held = place < (-(-length[children] // ps))[:, None]
    refs.index_add_(0, rows.clamp(min=0).flatten().long(), -held.flatten().to(torch.int32))
    table[children] = -1
    length[children] = 0
    return grown + [table, length, refs, pool]


def _plain_compact(s):
    s["table"].copy_(s["table0"])
    s["refs"].copy_(s["refs0"])
    table, refs, pool = s["table"], s["refs"], s["pool"]
    used = refs != 0
    place = torch.arange(refs.numel(), device="cuda")
    total = used.sum()
    source = torch.nonzero(used & (place >= total))[:, 0]
    target = torch.nonzero(~used & (place < total))[:, 0]
    pool[target] = pool[source]
    refs[target] = refs[source]
    refs[source] = 0
    now = place.to(torch.int32)
    now[source] = target.to(torch.int32)
    table.copy_(torch.where(table >= 0, now[table.clamp(min=0).long()], table))
    return [table, refs, pool]


def _plain_logprobs(s):
    raw, targets, k = s["logits"].float(), s["targets"], s["top"]
    x = raw * s["scale"]
    top = x.amax(1, keepdim=True).clamp(min=-3e38)
    away = (x - top).clamp_(min=-1e30)  # a masked token: probability 0, and 0 in the entropy
    e = torch.exp(away)
    empty = (raw == -math.inf).all(1, keepdim=True)
    e = e.masked_fill(empty, 0.0)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total.clamp(min=1e-38))
    entropy = (log_total - (e * away).sum(1, keepdim=True) / total.clamp(min=1e-38)).masked_fill(empty, 0.0)
    given = x.gather(1, targets.clamp(min=0)[:, None]) - top - log_total
    logprob = given.masked_fill(empty, -math.inf)[:, 0].masked_fill(targets < 0, 0.0)
    # value descending, index ascending: one key of both
    bits = (raw + 0.0).view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * (1 << 20)
    order = order - torch.arange(raw.shape[1], device="cuda")
    ids = torch.topk(order, k, dim=1)[1]
    chosen = (x.gather(1, ids) - top - log_total).masked_fill(empty, -math.inf)
    return [logprob, entropy[:, 0], ids, chosen]


# ------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    if case["kind"] in ("fork", "compact"):
        return None  # copies and whole numbers
    s = prepare(case, seed)
    if case["kind"] == "attend":
        n, hq, d = s["q"].shape
        group = hq // case["kv_heads"]
        out = torch.zeros(n, hq, d, dtype=torch.float64, device="cuda")
        lse = torch.full((n, hq), -math.inf, dtype=torch.float64, device="cuda")
        for i, count in enumerate(_lengths(case).tolist()):
            if not count:
                continue
            pages = s["table"][i, :-(-count // case["page_size"])].long()
            for g in range(case["kv_heads"]):
                kv = s["pool"][pages, s["layer"], :, g].double()  # [pages, 2, ps, d]
                keys, values = kv[:, 0].reshape(-1, d)[:count], kv[:, 1].reshape(-1, d)[:count]
                rows = slice(g * group, (g + 1) * group)
                z = s["q"][i, rows].double() @ keys.T * s["scale"]
                lse[i, rows] = torch.logsumexp(z, 1)
                out[i, rows] = torch.softmax(z, 1) @ values
        return [out, lse]
    outs = [[], [], []]
    k = case["top"]
    for a in range(0, case["rows"], 128):
        raw, t = s["logits"][a:a + 128].double(), s["targets"][a:a + 128]
        x = raw * case["scale"]
        logp = x - torch.logsumexp(x, 1, keepdim=True)
        none = torch.isneginf(raw).all(1, keepdim=True)
        logp = torch.where(none, torch.full_like(logp, -math.inf), logp)
        p = torch.exp(logp)
        outs[0].append(torch.where(t < 0, torch.zeros_like(logp[:, 0]), logp.gather(1, t.clamp(min=0)[:, None])[:, 0]))
        outs[1].append(-torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1))
        outs[2].append(torch.topk(logp, k, dim=1)[0])
    return [torch.cat(outs[0]), torch.cat(outs[1]), None, torch.cat(outs[2])]
