"""What a generating step runs between its matrix products -- residual sums with norms, drawn tokens, an 8-bit
cache -- against plain models: whole numbers exactly, numbers in 64 bits within bounds derived below."""
import numpy as np
import pytest
import torch

import answer_model
import step_model as model

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def copes():
    from paper_2608_02391_gb300 import copes as c
    c.load()
    return c


def ids(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def f64(t):
    return t.detach().double().cpu().numpy()


def error_bits(copes):
    """0, or the bits that copes_check reports (and clears)."""
    try:
        copes.check()
        return 0
    except copes.CopesError as e:
        assert e.code == copes.ERR_DEVICE_CHECK
        return int(str(e).split("bits 0x")[1].split(":")[0], 16)


# ------------------------------------------------------------------- residual sums and norms
def check_norm(got_s, got_h, x, weight, y, out_weight, gate, scale, eps):
    """With u the unit roundoff: outputs round to u of themselves.  A sum of squares adds, in a thread, up to 32
    squares (h / 1024 in rows that are read again), then over threads 10 and up to 32 warps: (74 + h / 1024) 2^-24 of
    itself at most, of which a root has half; the root's reciprocal and the division add 2^-22.  z has three more
    roundings, s one of its two terms and one of itself; what s is off by moves its norm by as much, and its
    rms by the 2-norm of that.  An s past the largest number of its type is infinite there (or not, within 2^-7 of
    it), and one past fp32 makes its norm NaN and the rest of its row's 0."""
    u = 2.0**-8 if x.dtype == torch.bfloat16 else 2.0**-24
    d = lambda t: None if t is None else f64(t)
    s, h = model.norm(d(x), d(weight), d(y), d(out_weight), d(gate), scale, eps)
    root = (74 + x.shape[1] / 1024) * 2.0**-25 + 2.0**-22
    off = 0.0 if y is None else np.abs(s - d(x)) * (root + 2.0**-22) + 2.0**-24 * (np.abs(s) + np.abs(d(x)))
    size, most = np.abs(s), torch.finfo(torch.float32).max
    near = np.abs(size / most - 1) <= 2.0**-7
    past = (size > most) & ~near
    if got_s is not None and y is not None:
        got = f64(got_s)
        assert np.array_equal(got[past], np.copysign(np.inf, s[past]))
        with np.errstate(invalid="ignore"):
            assert (near | past | (np.abs(got - s) <= 1.01 * u * size + off + 1e-38)).all()
    if got_h is not None:
        got = f64(got_h)
        rows = past.any(1)
        assert np.isnan(got[past]).all() and not got[rows][~past[rows] & ~near[rows]].any()
        rows |= near.any(1)
        rms = np.sqrt((s * s).mean(1, keepdims=True) + eps)
        moved = np.sqrt((np.square(off) * np.ones_like(s)).mean(1, keepdims=True)) / rms
        tol = np.abs(h) * (1.01 * u + root + 2.0**-22 + moved) + off / rms * np.abs(d(weight)) + 1e-38
        with np.errstate(invalid="ignore"):
            assert (rows[:, None] | (np.abs(got - h) <= tol)).all(), (np.abs(got - h) / tol)[~rows].max()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,hidden", [(1, 1), (3, 2), (70, 7), (33, 8), (5, 64), (129, 80), (1000, 128), (9, 255), (31, 256), (3, 257),
                                      (1, 896), (40, 900), (17, 1000), (2, 2560), (5, 2561), (6, 4096), (3, 8190), (2, 8200), (2, 16384),
                                      (2, 16387), (1, 70000)])
def test_norms_match_64_bits(copes, n, hidden, dtype):
    g = torch.Generator("cuda").manual_seed(hidden)
    rand = lambda *shape, mean=0.0, std=1.0: (torch.randn(*shape, device="cuda", generator=g) * std + mean).to(DT[dtype])
    w, ow = rand(hidden, mean=1.0, std=0.2), rand(hidden, mean=1.0, std=0.2)
    for shift in (0, 1, 2):  # rows that begin anywhere
        wide = [rand(n, hidden + shift * 5) for _ in range(3)]
        x, y, gate = (t[:, shift:shift + hidden] for t in wide)
        same, h = copes.residual_norm(x, w, eps=1e-5)
        assert same is x
        check_norm(None, h, x, w, None, None, None, 1.0, 1e-5)
        for args in (dict(), dict(out_weight=ow), dict(gate=gate[0].contiguous(), scale=0.7),
                     dict(out_weight=ow, gate=gate, scale=-0.3), dict(gate=gate)):
            s, h = copes.residual_norm(x, w, y=y, eps=1e-6, **args)
            full = {**dict(out_weight=None, gate=None, scale=1.0), **args}
            check_norm(s, h, x, w, y, full["out_weight"], full["gate"], full["scale"], 1e-6)
        s2, none = copes.residual_norm(x, None, y=y, eps=1e-6, **args)
        assert none is None and torch.equal(s2, s)
        s, h = copes.residual_norm(x, w, y=y, out_weight=ow, eps=1e-6)
        x2, y2 = x.clone(), y.clone()
        into = copes.residual_norm(x2, w, y=y2, out_weight=ow, eps=1e-6, out=x2, normed=y2)  # in place
        assert into[0] is x2 and into[1] is y2
        check_norm(x2, y2, x, w, y, ow, None, 1.0, 1e-6)
        out = torch.full((n, hidden + 3), 7.0, device="cuda", dtype=DT[dtype])  # rows of a wider buffer
        copes.residual_norm(x, w, y=y, out_weight=ow, eps=1e-6, out=out[:, 1:1 + hidden], normed=torch.empty_like(h))
        check_norm(out[:, 1:1 + hidden], None, x, w, y, ow, None, 1.0, 1e-6)
        assert (out[:, 0] == 7).all() and (out[:, 1 + hidden:] == 7).all()
    assert error_bits(copes) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hidden", [3, 96, 128, 1000, 20000])
def test_norms_of_extreme_rows(copes, hidden, dtype):
    """Zeros, squares past fp32 in some rows of a warp and not in others, squares below it, infinities and NaN."""
    n = 40
    x = torch.randn(n, hidden, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    x[3] = 0
    x[4] *= 1e30
    x[5] *= 2e37
    x[17] = 3e38
    x[18] *= 1e-25
    x[19] *= 1e-12
    x = x.to(DT[dtype])
    w = torch.linspace(0.5, 1.5, hidden, device="cuda").to(DT[dtype])
    for eps in (1e-6, 1e-30):
        _, h = copes.residual_norm(x, w, eps=eps)
        check_norm(None, h, x, w, None, None, None, 1.0, eps)
        s, h = copes.residual_norm(torch.zeros_like(x), w, y=x, out_weight=w, scale=2.0, eps=eps)
        check_norm(s, h, torch.zeros_like(x), w, x, w, None, 2.0, eps)
    assert not h[3].any()
    x[6, hidden // 2] = torch.inf
    x[7, 0] = torch.nan
    _, h = copes.residual_norm(x, w)
    assert torch.isnan(h[6, hidden // 2]) and torch.isnan(h[7]).all()
    rest = h[6].clone()
    rest[hidden // 2] = 0
    assert not rest.any() and torch.isfinite(h[[i for i in range(n) if i not in (6, 7)]]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,hidden", [(6100, 1032), (2600, 2560), (1900, 4096), (1250, 8192)])
def test_norms_of_many_rows(copes, n, hidden, dtype):
    """More rows than the GPU works on at once, among them ones whose squares are past fp32, in place too."""
    g = torch.Generator("cuda").manual_seed(n)
    rand = lambda *shape: torch.randn(*shape, device="cuda", generator=g)
    w, ow = (rand(hidden) * 0.2 + 1).to(DT[dtype]), (rand(hidden) * 0.2 + 1).to(DT[dtype])
    x, y, gate = (rand(n, hidden + 16).to(DT[dtype])[:, 8:8 + hidden] for _ in range(3))
    x[n // 2] = 2e38
    y[n - 3] = 3e38
    for args in (dict(out_weight=ow), dict(gate=gate[0].contiguous(), scale=0.7), dict(out_weight=ow, gate=gate, scale=-0.3)):
        full = {**dict(out_weight=None, gate=None, scale=1.0), **args}
        s, h = copes.residual_norm(x, w, y=y, eps=1e-6, **args)
        rows = torch.tensor(sorted({0, 1, 607, 608, 1216, n // 2, n - 3, n - 1} & set(range(n))) + list(range(5, n, 97)), device="cuda")
        token = full["gate"] if full["gate"] is None or full["gate"].dim() == 1 else full["gate"][rows]
        check_norm(s[rows], h[rows], x[rows], w, y[rows], full["out_weight"], token, full["scale"], 1e-6)
        x2, y2 = x.clone(), y.clone()
        copes.residual_norm(x2, w, y=y2, eps=1e-6, out=x2, normed=y2, **args)
        bits = lambda t: t.contiguous().view(torch.int16)  # NaN among them
        assert torch.equal(bits(x2), bits(s)) and torch.equal(bits(y2), bits(h))
        only, none = copes.residual_norm(x, None, y=y, eps=1e-6, **args)
        assert none is None and torch.equal(bits(only), bits(s))


def test_outputs_that_a_norm_would_not_write_are_refused(copes):
    x, w = torch.ones(2, 8, device="cuda"), torch.ones(8, device="cuda")
    for kw in (dict(out=x.clone()), dict(weight=None, y=x, normed=x.clone())):
        with pytest.raises(AssertionError):
            copes.residual_norm(**{**dict(x=x, weight=w), **kw})
    with pytest.raises(copes.CopesError):
        copes.residual_norm(x, None)  # nothing to write
    assert error_bits(copes) == 0


def test_norms_of_no_rows_and_of_rows_past_32_bits(copes):
    w = torch.ones(64, device="cuda", dtype=torch.bfloat16)
    s, h = copes.residual_norm(torch.empty(0, 64, device="cuda", dtype=torch.bfloat16), w,
                               y=torch.empty(0, 64, device="cuda", dtype=torch.bfloat16))
    assert s.shape == h.shape == (0, 64)
    x = torch.empty((1 << 32) + 64, device="cuda", dtype=torch.bfloat16).as_strided((3, 64), (1 << 31, 1))
    x.copy_(torch.randn(3, 64, device="cuda"))
    _, h = copes.residual_norm(x, w)
    check_norm(None, h, x, w, None, None, None, 1.0, 1e-6)


# ------------------------------------------------------------------------------ drawn tokens
def check_sample(copes, logits, u, expect_bits=0, **kw):
    """ids and counts exactly.  A log probability is a sum of two terms of one sign, each off by less than 2^-22."""
    kw = {**dict(top_k=0, top_p=1.0, min_p=0.0, scale=1.0), **kw}
    r = copes.sample_tokens(logits, u, **kw)
    assert error_bits(copes) == expect_bits
    x, uu = logits.detach().float().cpu().numpy(), u.cpu().numpy()
    got_ids, got_lp, got_kept = r.ids.cpu().numpy(), f64(r.logprob), r.kept.cpu().numpy()
    for i in range(len(x)):
        want, lp, kept = model.sample(x[i], float(uu[i]), kw["top_k"], kw["top_p"], kw["min_p"], float(np.float32(kw["scale"])))
        assert (got_ids[i], got_kept[i]) == (want, kept), (i, kw)
        if want < 0:
            assert np.isnan(got_lp[i])
        else:
            assert abs(got_lp[i] - lp) <= 2.0**-21 * abs(lp), (i, kw, got_lp[i], lp)
    return r


CUTS = [dict(), dict(top_k=1), dict(top_k=20), dict(top_p=0.9), dict(top_k=50, top_p=0.95), dict(min_p=0.05),
        dict(top_k=700, top_p=0.5, scale=0.6), dict(top_k=3000, min_p=0.001), dict(top_k=5000, top_p=0.99), dict(top_p=0.999, scale=1.7),
        dict(top_k=10, min_p=1.0), dict(top_p=1e-9)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,vocab", [(1, 1), (2, 2), (3, 7), (5, 31), (4, 300), (3, 1024), (7, 4095), (2, 32003), (33, 32003), (1, 151936),
                                     (6, 151936), (20, 151936), (90, 10007), (400, 1031)])
def test_drawn_tokens_follow_the_definition(copes, n, vocab, dtype):
    g = torch.Generator("cuda").manual_seed(vocab + n)
    wide = torch.randn(n, vocab + 3, device="cuda", generator=g) * (1.0 + 3.0 * torch.rand(n, 1, device="cuda", generator=g))
    wide[:, ::max(1, vocab // 9)] += 9.0 * torch.rand(n, 1, device="cuda", generator=g)
    wide = wide.to(DT[dtype])
    u = torch.rand(n, device="cuda", generator=g)
    u[0] = 0.0
    u[-1] = 1 - 2.0**-24
    for i, kw in enumerate(CUTS):
        logits = wide[:, :vocab].contiguous() if i % 3 == 0 else wide[:, i % 3:i % 3 + vocab]  # rows that begin anywhere
        check_sample(copes, logits, u, **kw)


def special_rows(vocab, dtype):
    """Rows that cuts can go wrong at, for a lowest value of the type."""
    g = torch.Generator("cuda").manual_seed(vocab)
    up = torch.arange(vocab, device="cuda", dtype=torch.float32) / vocab * 20 - 10
    low = torch.finfo(DT[dtype]).min
    few = torch.full((vocab,), -torch.inf, device="cuda")
    few[[0, vocab // 2, vocab - 1]] = torch.tensor([1.0, 2.0, 2.0], device="cuda")
    last = torch.full((vocab,), -torch.inf, device="cuda")
    last[-1] = -50.0
    zeros = torch.zeros(vocab, device="cuda")
    zeros[::2] = -0.0
    block = torch.full((vocab,), -3.0, device="cuda")
    block[vocab // 3:vocab // 3 + 200] = 4.0 + torch.arange(min(200, vocab - vocab // 3), device="cuda") / 512
    lows = torch.full((vocab,), low, device="cuda")
    lows[vocab // 2] = 3.0
    one = torch.zeros(vocab, device="cuda")
    one[vocab // 3] = 300.0
    steps = torch.floor(torch.rand(vocab, device="cuda", generator=g) * 3)
    two = torch.where(torch.rand(vocab, device="cuda", generator=g) < 0.5, 5.0, -25.0)
    near = torch.randn(vocab, device="cuda", generator=g) * 1e-3
    return [up, up.flip(0), torch.full((vocab,), 1.5, device="cuda"), torch.full((vocab,), -torch.inf, device="cuda"), few, last, zeros,
            block, lows, torch.full((vocab,), low, device="cuda"), torch.full((vocab,), -low, device="cuda"), one, steps, two, near,
            torch.where(torch.rand(vocab, device="cuda", generator=g) < 0.9, -torch.inf, up)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [5, 300, 9001, 70001])
@pytest.mark.parametrize("copies", [1, 12])
def test_drawn_tokens_of_ties_masks_and_orders(copes, vocab, dtype, copies):
    """Few rows, each by a cluster of blocks, and many, each by one."""
    logits = torch.stack(special_rows(vocab, dtype) * copies).to(DT[dtype])
    u = torch.rand(len(logits), device="cuda", generator=torch.Generator("cuda").manual_seed(vocab))
    for kw in CUTS[::1 if copies == 1 else 3]:
        check_sample(copes, logits, u, **kw)
    check_sample(copes, logits, u, scale=1e-3, top_p=0.7)
    check_sample(copes, logits, u, scale=50.0, top_p=0.7)
    check_sample(copes, logits, u, top_k=vocab, top_p=0.7)


def test_drawn_tokens_of_rows_that_nothing_can_be_drawn_from(copes):
    x = torch.randn(7, 999, device="cuda")
    x[1, 5] = torch.nan
    x[2, 998] = torch.inf
    x[3] = torch.nan
    x[4] = -torch.inf
    for dtype in DT.values():
        u = torch.full((7,), 0.5, device="cuda")
        for kw in (dict(), dict(top_k=5), dict(top_p=0.5)):
            r = check_sample(copes, x.to(dtype), u, expect_bits=32, **kw)
            assert r.ids.cpu().tolist().count(-1) == 4
    u = torch.tensor([0.0, 1.0, -0.1, torch.nan, torch.inf, 0.999, -0.0], device="cuda")
    check_sample(copes, torch.randn(7, 999, device="cuda"), u, expect_bits=32)
    check_sample(copes, x[4:5], u[:1])  # a row that is masked wholly is no error
    r = copes.sample_tokens(x[:0], u[:0])
    assert r.ids.numel() == 0 and error_bits(copes) == 0


def test_a_top_k_past_32_bits_keeps_all(copes):
    logits, u = torch.randn(3, 500, device="cuda"), torch.rand(3, device="cuda")
    for top_k in (500, 2**31, 2**32, 2**32 + 5):
        assert copes.sample_tokens(logits, u, top_k=top_k).kept.tolist() == [500] * 3
    for top_k in (-1, -2**32):
        with pytest.raises(copes.CopesError):
            copes.sample_tokens(logits, u, top_k=top_k)


def test_drawn_tokens_do_not_depend_on_the_batch(copes):
    """A row alone, by a cluster of eight blocks, and among hundreds, by one."""
    g = torch.Generator("cuda").manual_seed(8)
    logits = (torch.randn(300, 50021, device="cuda", generator=g) * 2).bfloat16()
    u = torch.rand(300, device="cuda", generator=g)
    for kw in (dict(), dict(top_p=0.9), dict(top_k=40), dict(top_k=4000)):
        many = copes.sample_tokens(logits, u, **kw)
        for i in (0, 7, 299):
            alone = copes.sample_tokens(logits[i:i + 1], u[i:i + 1], **kw)
            assert alone.ids[0] == many.ids[i] and alone.kept[0] == many.kept[i] and alone.logprob[0] == many.logprob[i]
    assert error_bits(copes) == 0


def test_drawn_tokens_of_a_large_vocabulary_and_of_rows_past_32_bits(copes):
    for dtype in DT.values():
        x = (torch.randn(2, 4_000_000, device="cuda", generator=torch.Generator("cuda").manual_seed(2)) * 2).to(dtype)
        u = torch.tensor([0.3, 0.99], device="cuda")
        for kw in (dict(), dict(top_k=100, top_p=0.9), dict(top_p=0.8)):
            check_sample(copes, x, u, **kw)
    row = 1 << 31
    x = torch.empty(2 * row + 400, device="cuda", dtype=torch.bfloat16).as_strided((3, 400), (row, 1))
    x.copy_(torch.randn(3, 400, device="cuda"))
    check_sample(copes, x, torch.tensor([0.1, 0.5, 0.9], device="cuda"), top_p=0.9)


# ------------------------------------------------------------------------------ 8-bit cache
def cache8(copes, lens, layers, kv, ps, d, seed=0, spare=3, poison=True):
    """An 8-bit cache of these lengths with pages in random order and random codes; what no token owns is NaN."""
    rng = np.random.default_rng(seed)
    pages = [-(-int(x) // ps) for x in lens]
    n_pages = sum(pages) + spare
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((len(lens), max(max(pages), 1) + 1), -1, np.int32)
    refs = np.zeros(n_pages, np.int32)
    codes = rng.integers(0, 127, (n_pages, layers, 2, kv, ps, d)) + 128 * rng.integers(0, 2, (n_pages, layers, 2, kv, ps, d))
    powers = rng.integers(116, 122, (n_pages, layers, 2, kv, ps))
    used = np.zeros((n_pages, ps), bool)
    at = 0
    for i, p in enumerate(pages):
        table[i, :p] = order[at:at + p]
        refs[table[i, :p]] = 1
        for j in range(p):
            used[table[i, j], :min(ps, int(lens[i]) - j * ps)] = True
        at += p
    if poison:
        codes = np.where(used[:, None, None, None, :, None], codes, 127)
    pool = np.full((n_pages, layers, copes.KVCache.layer_bytes(kv, ps, d)), 0xAB, np.uint8)
    size = 2 * kv * ps * d
    pool[:, :, :size] = codes.reshape(n_pages, layers, -1)
    pool[:, :, size:size + 2 * kv * ps] = powers.reshape(n_pages, layers, -1)
    t = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()
    return copes.KVCache(torch.from_numpy(pool).cuda(), t(table), t(lens), t(refs), heads=(kv, ps, d))


def values_of(cache, layer):
    """[n_pages, 2, kv, ps, d] in float64."""
    kv, ps, d = cache.heads
    raw, size = cache.pool[:, layer].cpu().numpy(), 2 * kv * ps * d
    return model.held(raw[:, :size].reshape(-1, 2, kv, ps, d), raw[:, size:size + 2 * kv * ps].reshape(-1, 2, kv, ps))


def check_attention(cache, layer, q, slots, scale, out, lse):
    """Against 64 bits: the output rounds to 2^-8 |o|.  A score's error, d + 6 roundings or cuts of 2^-23 of
    S = sum |scale q k| and 2^-36 of it for what fp16 does not hold of q, moves each weight twice; weights in two
    fp16 terms lose 2^-21 and 2^-39 of the tile's largest weighted unit, exp 2^-20, sums of L terms 8 sqrt(L) 2^-24."""
    d, ps = cache.desc.head_dim, cache.desc.page_size
    values, table, length = values_of(cache, layer), cache.table.cpu().numpy(), cache.length.cpu().numpy()
    qd, got, got_lse = f64(q), f64(out), f64(lse)
    for i, s in enumerate(slots):
        n = int(length[s])
        rows = values[table[s, :-(-n // ps)]] if n else np.zeros((0,) + values.shape[1:])
        keys = rows[:, 0].transpose(0, 2, 1, 3).reshape(-1, values.shape[2], d)[:n]
        vals = rows[:, 1].transpose(0, 2, 1, 3).reshape(-1, values.shape[2], d)[:n]
        o, l, mass, size = answer_model.attention(qd[i], keys, vals, scale)
        if n == 0:
            assert not got[i].any() and np.isneginf(got_lse[i]).all()
            continue
        score = (d + 6) * 2.0**-23 * size
        rel = 2 * score + 2.0**-19 + 8 * np.sqrt(n) * 2.0**-24
        tol = 1.01 * 2.0**-8 * np.abs(o) + rel[:, None] * mass + 2.0**-30 * mass.max(1, keepdims=True) + 1e-38
        assert np.isfinite(got[i]).all() and (np.abs(got[i] - o) <= tol).all(), (i, n, (np.abs(got[i] - o) / tol).max())
        tol = score + 2.0**-20 + 8 * np.sqrt(n) * 2.0**-24 + 2.0**-23 * np.abs(l)
        assert (np.abs(got_lse[i] - l) <= tol).all(), (i, n)


SHAPES = [  # q heads, kv heads, head_dim, page size
    (14, 2, 64, 16), (32, 8, 128, 16), (4, 4, 64, 1), (15, 5, 80, 7), (16, 1, 128, 64), (9, 1, 96, 50), (24, 3, 128, 33),
    (40, 1, 64, 16), (12, 4, 256, 16), (17, 1, 256, 8), (3, 3, 16, 5), (8, 2, 48, 128), (33, 1, 144, 16), (8, 4, 192, 16)]


@pytest.mark.parametrize("heads,kv,d,ps", SHAPES)
def test_attention_over_8_bits(copes, heads, kv, d, ps):
    lens = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 0, 300, 1000, 31, 777]
    cache = cache8(copes, lens, 2, kv, ps, d, seed=heads + d)
    n = len(lens)
    qkv = (torch.randn(n, heads + 3, d + 5, device="cuda") * 1.5).bfloat16()
    q = qkv[:, 2:2 + heads, :d]  # strides of rows and heads are not the shape's
    for layer in (0, 1):
        out, lse = copes.paged_attention(cache, layer, q, scale=0.1 * d ** -0.5)
        check_attention(cache, layer, q, range(n), 0.1 * d ** -0.5, out, lse)
    slots = [13, 0, 14, 14, 3, 16]
    out, lse = copes.paged_attention(cache, 1, q[:6], slots=ids(slots), scale=0.01)
    check_attention(cache, 1, q[:6], slots, 0.01, out, lse)
    assert error_bits(copes) == 0


@pytest.mark.parametrize("n,longest,heads,kv,d,ps", [(1, 20011, 32, 8, 128, 16), (1, 9001, 2, 1, 64, 16), (3, 7013, 14, 2, 64, 7),
                                                     (200, 90, 4, 2, 64, 16), (2, 4099, 12, 4, 256, 48), (1000, 60, 4, 2, 64, 16),
                                                     (420, 150, 12, 4, 128, 16), (500, 1000, 12, 4, 80, 16), (470, 900, 24, 8, 64, 7)])
def test_attention_over_8_bits_of_long_and_many_sequences(copes, n, longest, heads, kv, d, ps):
    rng = np.random.default_rng(n)
    lens = rng.integers(0, min(longest, 200) + 1 if n > 100 else longest + 1, n)
    lens[-1] = longest
    cache = cache8(copes, lens, 1, kv, ps, d, seed=n)
    q = (torch.randn(n, heads, d, device="cuda") * 3).bfloat16()
    scale = 0.1 * d ** -0.5
    first = copes.paged_attention(cache, 0, q, scale=scale)
    check_attention(cache, 0, q, range(n), scale, *first)
    for _ in range(3):  # joined in one order: the same bits again, on the same workspace
        again = copes.paged_attention(cache, 0, q, scale=scale)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    assert error_bits(copes) == 0


def test_attention_over_8_bits_of_extreme_units(copes):
    """Tokens whose keys or values are larger than others' by powers of two of any size, tiny and huge queries."""
    d, ps = 64, 16
    rng = np.random.default_rng(4)
    for span in (3, 20, 60):
        lens = [1, 16, 40, 333]
        cache = cache8(copes, lens, 1, 2, ps, d, seed=span, poison=False)
        size = 2 * 2 * ps * d
        powers = rng.integers(127 - span, 128, (cache.desc.n_pages, 1, 2, 2, ps))
        powers[:, :, 0] = np.minimum(powers[:, :, 0], 118)
        cache.pool[:, :, size:size + 4 * ps] = torch.from_numpy(powers.reshape(cache.desc.n_pages, 1, -1).astype(np.uint8)).cuda()
        for size_q in (1.0, 2.0**-60, 2.0**60):
            q = (torch.randn(4, 6, d, device="cuda") * size_q).bfloat16()
            q[:, 0] = 0
            q[:, 1, 5:] *= 2.0**-20
            scale = 2.0**-6 / size_q
            check_attention(cache, 0, q, range(4), scale, *copes.paged_attention(cache, 0, q, scale=scale))
    q[0, 2, 3] = torch.inf
    q[1, 3, 4] = torch.nan
    out, lse = copes.paged_attention(cache, 0, q, scale=2.0**-6)
    assert not torch.isfinite(out[0, 2]).any() and torch.isnan(out[1, 3]).all() and torch.isnan(lse[1, 3])
    assert torch.isfinite(out[0, [0, 1, 4, 5]]).all()
    assert error_bits(copes) == 0


@pytest.mark.parametrize("d", [64, 128, 256])
def test_bytes_past_a_sequence_are_not_read(copes, d):
    cache = cache8(copes, [3, 33], 1, 2, 16, d, seed=d, spare=0, poison=False)
    q = torch.randn(2, 4, d, device="cuda").bfloat16()
    out, lse = copes.paged_attention(cache, 0, q, scale=0.01)
    size, table = 2 * 2 * 16 * d, cache.table.tolist()
    for page, begin in ((table[0][0], 3), (table[1][2], 1)):
        cache.pool[page, 0, :size].view(4, 16, d)[:, begin:] = 0xFF
        cache.pool[page, 0, size:size + 64].view(4, 16)[:, begin:] = 0xFF
    again = copes.paged_attention(cache, 0, q, scale=0.01)
    assert torch.isfinite(out).all() and torch.equal(again[0], out) and torch.equal(again[1], lse)
    assert error_bits(copes) == 0


@pytest.mark.parametrize("kv,d,ps", [(2, 64, 16), (3, 16, 5), (5, 80, 7), (8, 128, 16), (1, 256, 33), (2, 48, 1)])
def test_what_is_written_in_8_bits_is_read_back(copes, kv, d, ps):
    layers, lens = 3, [0, 1, ps, ps + 1, 5 * ps + 2, 40]
    cache = cache8(copes, lens, layers, kv, ps, d, seed=d)
    rng = np.random.default_rng(d)
    rows = [(s, t) for s in range(len(lens)) for t in range(lens[s])]
    rows = [rows[i] for i in rng.permutation(len(rows))[:150]]
    n = len(rows)
    qkv = torch.randn(n, 3, kv, d, device="cuda") * 10.0 ** torch.randint(-30, 30, (n, 1, 1, 1), device="cuda")
    qkv[0] = 0
    qkv[1, :, 0, 3] = torch.inf
    qkv[2, :, -1, 0] = torch.nan
    qkv[3] = 1e-41
    qkv[4, :, :, 1] = 3.3e38
    qkv[5, :, :, ::2] = -0.0
    qkv = qkv.bfloat16()
    before = cache.pool.clone()
    slots, position = ids(s for s, _ in rows), ids(t for _, t in rows)
    copes.cache_append(cache, 1, qkv[:, 1], qkv[:, 2], slots=slots, position=position)
    k, v = copes.cache_read(cache, 1, slots=slots, position=position)
    assert error_bits(copes) == 0
    size = 2 * kv * ps * d
    raw, table = cache.pool[:, 1].cpu().numpy(), cache.table.cpu().numpy()
    codes, powers = raw[:, :size].reshape(-1, 2, kv, ps, d), raw[:, size:size + 2 * kv * ps].reshape(-1, 2, kv, ps)
    for which, got in ((0, k), (1, v)):
        x = f64(qkv[:, 1 + which])
        values, code, power = model.stored(x)
        rounded = f64(torch.from_numpy(values).bfloat16())  # bf16 holds 2^-133 and more of them exactly
        assert np.array_equal(f64(got), rounded, equal_nan=True)
        for r, (s, t) in enumerate(rows):
            page, place = table[s, t // ps], t % ps
            assert np.array_equal(powers[page, which, :, place], power[r])
            there = codes[page, which, :, place]
            assert np.array_equal(there[code[r] >= 0], code[r][code[r] >= 0]) and ((there[code[r] < 0] & 127) == 127).all()
    after = cache.pool.clone()  # nothing else was written
    at = torch.zeros_like(after, dtype=torch.bool)[:, 1]
    mark_c, mark_p = np.zeros_like(codes, dtype=bool), np.zeros_like(powers, dtype=bool)
    for s, t in rows:
        mark_c[table[s, t // ps], :, :, t % ps] = True
        mark_p[table[s, t // ps], :, :, t % ps] = True
    at[:, :size] = torch.from_numpy(mark_c.reshape(len(raw), -1)).cuda()
    at[:, size:size + 2 * kv * ps] = torch.from_numpy(mark_p.reshape(len(raw), -1)).cuda()
    assert torch.equal(after[:, [0, 2]], before[:, [0, 2]]) and torch.equal(after[:, 1][~at], before[:, 1][~at])
    # rows from anywhere, and the default: every slot's last token
    odd = torch.empty(n, kv, d + 1, device="cuda", dtype=torch.bfloat16)
    odd[:, :, 1:] = qkv[:, 1]
    copes.cache_append(cache, 1, odd[:, :, 1:], odd[:, :, 1:], slots=slots, position=position)
    assert torch.equal(cache.pool[:, 1, :size].view(-1, 2, size // 2)[:, 0], after[:, 1, :size].view(-1, 2, size // 2)[:, 0])
    last = copes.cache_read(cache, 1)
    assert error_bits(copes) == 32 and not last[0][0].any()  # slot 0 has no token
    want = copes.cache_read(cache, 1, slots=ids(range(1, 6)), position=ids(x - 1 for x in lens[1:]))
    assert torch.equal(last[0][1:].view(torch.int16), want[0].view(torch.int16))


def test_rows_that_name_one_token_of_8_bits(copes):
    """Equal ones are kept, of others each code and byte is one of theirs; read, each gives the token."""
    cache = cache8(copes, [20, 20], 1, 2, 16, 64, seed=1)
    x = (torch.randn(300, 2, 2, 64, device="cuda") * 2.0 ** torch.randint(-5, 5, (300, 1, 1, 1), device="cuda")).bfloat16()
    x[150:] = x[150]
    slots, position = ids([0] * 150 + [1] * 150), ids([7] * 150 + [19] * 150)
    copes.cache_append(cache, 0, x[:, 0], x[:, 1], slots=slots, position=position)
    k, v = copes.cache_read(cache, 0, slots=slots, position=position)
    assert torch.equal(k, k[[0] * 150 + [150] * 150]) and torch.equal(v, v[[0] * 150 + [150] * 150])
    assert np.array_equal(f64(k[150]), model.stored(f64(x[150, 0]))[0]) and np.array_equal(f64(v[150]), model.stored(f64(x[150, 1]))[0])
    size, page = 2 * 2 * 16 * 64, int(cache.table[0, 0])
    raw = cache.pool[page, 0].cpu().numpy()
    for which in (0, 1):
        _, code, power = model.stored(f64(x[:150, which]))
        there, byte = raw[:size].reshape(2, 2, 16, 64)[which, :, 7], raw[size:size + 64].reshape(2, 2, 16)[which, :, 7]
        assert (code == there).any(0).all() and (power == byte).any(0).all()
    assert error_bits(copes) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_reading_back_other_caches(copes, dtype):
    cache = copes.KVCache.empty(12, 2, 3, 4, 24, 4, 3, dtype=DT[dtype])
    cache.pool.normal_()
    copes.cache_grow(cache, ids([0, 1, 2]), ids([5, 1, 12]))
    kv = torch.randn(18, 2, 3, 24, device="cuda").to(DT[dtype])
    slots, position = ids([0] * 5 + [1] + [2] * 12), ids(list(range(5)) + [0] + list(range(12)))
    copes.cache_append(cache, 1, kv[:, 0], kv[:, 1], slots=slots, position=position)
    k, v = copes.cache_read(cache, 1, slots=slots, position=position)
    assert torch.equal(k, kv[:, 0]) and torch.equal(v, kv[:, 1]) and error_bits(copes) == 0
    k, v = copes.cache_read(cache, 1, slots=ids([0, 3, 9, 2, -1, 1]), position=ids([4, 0, 0, 12, 0, -1]))
    assert error_bits(copes) == 32 and torch.equal(k[0], kv[4, 0]) and not k[1:].any() and not v[1:].any()
    cache.table[0, 0] = 99
    k, v = copes.cache_read(cache, 1, slots=ids([0, 0]), position=ids([0, 4]))
    assert error_bits(copes) == 32 and not k[0].any() and torch.equal(v[1], kv[4, 1])


def test_pages_of_8_bits_are_grown_forked_freed_and_moved(copes):
    """The bookkeeping of random calls, and whole pages, exponents among them, where they are copied."""
    kv, ps, d, layers, n_pages, slots, width = 3, 5, 48, 2, 30, 10, 6
    cache = copes.KVCache.empty(n_pages, layers, kv, ps, d, slots, width, dtype=torch.float8_e4m3fn)
    cache.pool.random_(0, 120)
    m, pool = answer_model.CacheModel(n_pages, ps, slots, width), cache.pool.clone()
    rng = np.random.default_rng(7)
    for _ in range(60):
        what, n = rng.choice(["grow", "fork", "free", "compact"]), int(rng.integers(1, 4))
        m.copies = []
        if what == "grow":
            s, add = rng.permutation(slots)[:n].tolist(), rng.integers(0, 9, n).tolist()
            copes.cache_grow(cache, ids(s), ids(add))
            bad = m.grow(s, add)
        elif what == "fork":
            children = rng.permutation(slots)[:n].tolist()
            parents = rng.choice(slots, n).tolist()
            copes.cache_fork(cache, ids(parents), ids(children))
            bad = m.fork(parents, children)
        elif what == "free":
            s = rng.permutation(slots)[:n].tolist()
            copes.cache_free(cache, ids(s))
            bad = m.free(s)
        else:
            copes.cache_compact(cache)
            m.compact()
            bad = 0
        for a, b in m.copies:
            pool[b] = pool[a]
        assert error_bits(copes) == bad
        assert cache.length.tolist() == m.length and cache.refs.tolist() == m.refs
        assert np.array_equal(cache.table.cpu().numpy(), m.table()) and torch.equal(cache.pool, pool)


def test_an_8_bit_cache_past_32_bits(copes):
    """Pages whose bytes start past 2^32 of the pool."""
    kv, ps, d = 2, 16, 128
    layer = copes.KVCache.layer_bytes(kv, ps, d)
    n_pages = (1 << 32) // layer + 40
    pool = torch.empty(n_pages, 1, layer, device="cuda", dtype=torch.uint8)
    cache = copes.KVCache(pool, torch.full((1, 8), -1, dtype=torch.int32, device="cuda"), ids([0]),
                          torch.zeros(n_pages, dtype=torch.int32, device="cuda"), heads=(kv, ps, d))
    cache.refs[:n_pages - 5] = 1
    copes.cache_grow(cache, ids([0]), 70)
    x = torch.randn(70, 2, kv, d, device="cuda").bfloat16()
    copes.cache_append(cache, 0, x[:, 0], x[:, 1], slots=ids([0] * 70), position=ids(range(70)))
    q = torch.randn(1, 8, d, device="cuda").bfloat16()
    out, lse = copes.paged_attention(cache, 0, q)
    small = copes.KVCache(pool[-5:].clone(), ids([0, 1, 2, 3, 4])[None].contiguous(), ids([70]), ids([1] * 5), heads=(kv, ps, d))
    check_attention(small, 0, q, [0], d ** -0.5, out, lse)
    k, _ = copes.cache_read(cache, 0, slots=ids([0] * 70), position=ids(range(70)))
    assert np.array_equal(f64(k), model.stored(f64(x[:, 0]))[0])
    assert error_bits(copes) == 0


# ------------------------------------------------------------------------------ together
def test_a_step_on_a_stream_and_in_a_graph(copes):
    """The calls of a generating step one after the other, on a side stream and replayed."""
    g = torch.Generator("cuda").manual_seed(9)
    rand = lambda *shape: torch.randn(*shape, device="cuda", generator=g).bfloat16()
    n, kv, d, hidden, vocab = 5, 2, 64, 128, 5000
    x, y, w = rand(n, hidden), rand(n, hidden), rand(hidden)
    k, v, head, rows = rand(n, kv, d), rand(n, kv, d), rand(vocab, hidden), ids(range(n))
    u = torch.rand(n, device="cuda", generator=g)

    def fresh():
        return cache8(copes, [3, 16, 17, 200, 1], 2, kv, 16, d, seed=2, spare=40, poison=False)

    def step(cache, stream=None):
        s, h = copes.residual_norm(x, w, y=y, out_weight=w, stream=stream)
        copes.cache_append(cache, 1, k, v, slots=rows, stream=stream)
        read = copes.cache_read(cache, 1, slots=rows, stream=stream)
        out, lse = copes.paged_attention(cache, 1, h.view(n, kv, d), slots=rows, stream=stream)
        s2, h2 = copes.residual_norm(s, w, y=out.flatten(1), stream=stream)
        if stream is None:
            r = copes.sample_tokens(h2 @ head.T, u, top_p=0.9)
        else:
            with torch.cuda.stream(stream):
                r = copes.sample_tokens(h2 @ head.T, u, top_p=0.9)
        return [s, h, *read, out, lse, s2, h2, r.ids, r.logprob, r.kept, cache.pool]

    want = step(fresh())
    side = torch.cuda.Stream()
    cache = fresh()
    side.wait_stream(torch.cuda.current_stream())
    got = step(cache, side)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    cache = fresh()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(cache)
    for _ in range(3):
        for t in held[:-1]:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b)
    assert error_bits(copes) == 0
