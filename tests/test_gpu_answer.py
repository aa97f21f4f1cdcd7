"""The operators that answer with the weights -- cache pages, paged attention, token log
probabilities -- against plain models: bookkeeping exactly, numbers in 64 bits within bounds
derived below."""
import numpy as np
import pytest
import torch

import answer_model as model

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


# ------------------------------------------------------------------------------ pages
def same(cache, m, pool):
    assert np.array_equal(cache.length.cpu().numpy(), m.length)
    assert np.array_equal(cache.refs.cpu().numpy(), m.refs)
    assert np.array_equal(cache.table.cpu().numpy(), m.table())
    assert torch.equal(cache.pool, pool)


@pytest.mark.parametrize("page_size,layers,kv,d,dtype,n_pages", [
    (16, 2, 2, 64, "bf16", 40), (1, 1, 1, 8, "bf16", 70), (7, 3, 5, 80, "fp32", 33), (50, 1, 3, 24, "bf16", 3000)])
def test_pages_follow_the_model_through_random_calls(copes, page_size, layers, kv, d, dtype, n_pages):
    rng = np.random.default_rng(page_size)
    slots, width = 12, 9
    cache = copes.KVCache.empty(n_pages, layers, kv, page_size, d, slots, width, dtype=DT[dtype])
    cache.pool.copy_(torch.randn(cache.pool.shape, device="cuda"))
    if n_pages > 2048:  # pages in use past one round of the search for free ones
        cache.refs[:2500] = 1
    m = model.CacheModel(n_pages, page_size, slots, width)
    m.refs = cache.refs.cpu().tolist()
    pool = cache.pool.clone()
    seen = set()
    for step in range(120):
        what = rng.choice(["grow", "fork", "free", "compact", "append", "copy"], p=[.35, .2, .15, .1, .15, .05])
        n = int(rng.integers(0, 6))
        bad = 0
        if what == "grow":
            s = rng.choice(slots, n, replace=bool(rng.random() < 0.1)).tolist()
            add = rng.integers(0, 3 * page_size + 2, n).tolist()
            if rng.random() < 0.1 and n:
                s[0] = int(rng.choice([-1, slots, 1 << 30]))
            if rng.random() < 0.3 and n:
                add = [add[0]] * n
                copes.cache_grow(cache, ids(s), add[0])
            else:
                copes.cache_grow(cache, ids(s), ids(add))
            bad = m.grow(s, add)
        elif what == "fork":
            empty = [i for i in range(slots) if not m.length[i]]
            children = rng.permutation(empty)[:n].tolist() if rng.random() < 0.8 else rng.choice(slots, n).tolist()
            parents = rng.choice(slots, len(children)).tolist()
            copes.cache_fork(cache, ids(parents), ids(children))
            bad = m.fork(parents, children)
            for a, b in m.copies:
                pool[b] = pool[a]
        elif what == "free":
            s = rng.integers(-1 if rng.random() < 0.2 else 0, slots, n).tolist()
            copes.cache_free(cache, ids(s))
            bad = m.free(s)
        elif what == "compact":
            counts = ids([-1, -1])
            copes.cache_compact(cache, counts)
            used = m.compact()
            assert counts.tolist() == list(used)
            for a, b in m.copies:
                pool[b] = pool[a]
        elif what == "append":
            s = [i for i in range(slots) if m.length[i]]
            layer = int(rng.integers(layers))
            pos = [int(rng.integers(m.length[i])) for i in s]
            if rng.random() < 0.5:
                pos = [m.length[i] - 1 for i in s]
            kvt = torch.randn(len(s), kv, 3, d, device="cuda", dtype=torch.float32).to(DT[dtype])
            copes.cache_append(cache, layer, kvt[:, :, 0], kvt[:, :, 2], slots=ids(s),
                               position=None if pos == [m.length[i] - 1 for i in s] else ids(pos))
            owner = {}
            for r, (i, p) in enumerate(zip(s, pos)):
                owner.setdefault((m.pages[i][p // page_size], p % page_size), []).append(r)
            for (page, place), rows in owner.items():
                got = cache.pool[page, layer, :, :, place]
                if len(rows) > 1:  # a shared page's token, written by each of its slots: value by value, one of theirs
                    theirs = kvt[rows][:, :, [0, 2]].transpose(1, 2)
                    assert (got == theirs).any(0).all()
                    pool[page, layer, :, :, place] = got
                else:
                    pool[page, layer, 0, :, place] = kvt[rows[0], :, 0]
                    pool[page, layer, 1, :, place] = kvt[rows[0], :, 2]
        else:
            perm = rng.permutation(n_pages)[:6].tolist()
            copes.cache_copy_pages(cache, ids(perm[:3]), ids(perm[3:]))
            for a, b in zip(perm[:3], perm[3:]):
                pool[b] = pool[a]
        assert error_bits(copes) == bad, (step, what)
        seen.add((what, bad))
        same(cache, m, pool)
    assert len(seen) >= 6


def test_grow_and_fork_change_all_or_nothing(copes):
    cache = copes.KVCache.empty(6, 1, 1, 4, 8, 5, 3)
    m = model.CacheModel(6, 4, 5, 3)
    cache.pool.normal_()
    pool = cache.pool.clone()
    for slots, add in [([0, 1], [5, 3]), ([1, 2], [9, 1]), ([2], [-1]), ([0, 0], [1, 1]), ([3, 5], [1, 1]), ([3, -1], [1, 1]),
                       ([2, 3], [8, 5]), ([0], [2**31 - 1]), ([2], [0])]:
        copes.cache_grow(cache, ids(slots), ids(add))
        assert error_bits(copes) == m.grow(slots, add)
        same(cache, m, pool)
    for parents, children in [([0], [0]), ([0, 2], [2, 3]), ([0, 0], [3, 3]), ([0], [1]), ([7], [2]), ([0], [5]), ([0, 1, 0], [2, 3, 4]),
                              ([0, 1], [2, 3])]:
        copes.cache_fork(cache, ids(parents), ids(children))
        assert error_bits(copes) == m.fork(parents, children)
        for a, b in m.copies:
            pool[b] = pool[a]
        same(cache, m, pool)


def test_a_long_prompt_and_many_children(copes):
    """Page lists longer than a block of the plan, refs raised from many blocks at once."""
    cache = copes.KVCache.empty(6000, 1, 1, 2, 8, 300, 2600)
    m = model.CacheModel(6000, 2, 300, 2600)
    cache.pool.normal_()
    pool = cache.pool.clone()
    copes.cache_grow(cache, ids([7, 3]), ids([5001, 2]))
    assert m.grow([7, 3], [5001, 2]) == 0
    children = [i for i in range(300) if i not in (3, 7)]
    copes.cache_fork(cache, ids([7] * len(children)), ids(children))
    assert m.fork([7] * len(children), children) == 0
    for a, b in m.copies:
        pool[b] = pool[a]
    assert error_bits(copes) == 0
    same(cache, m, pool)
    copes.cache_free(cache, ids([7] + children[::2] + [7]))
    m.free([7] + children[::2])
    copes.cache_compact(cache)
    m.compact()
    for a, b in m.copies:
        pool[b] = pool[a]
    assert error_bits(copes) == 0
    same(cache, m, pool)


def test_large_pages_are_copied_whole(copes):
    """Pages of several jobs, the last of them partly filled, and more jobs than blocks."""
    cache = copes.KVCache.empty(420, 30, 2, 5, 256, 210, 4)
    m = model.CacheModel(420, 5, 210, 4)
    cache.pool.normal_()
    pool = cache.pool.clone()

    def follow():
        for a, b in m.copies:
            pool[b] = pool[a]
        assert error_bits(copes) == 0
        same(cache, m, pool)

    parents = [0, 1, 2]
    copes.cache_grow(cache, ids(parents), ids([7, 5, 19]))
    assert m.grow(parents, [7, 5, 19]) == 0
    children = list(range(3, 210))
    of = [parents[i * 3 // len(children)] for i in range(len(children))]
    copes.cache_fork(cache, ids(of), ids(children))
    assert m.fork(of, children) == 0
    follow()
    copes.cache_free(cache, ids(children[:100]))
    m.free(children[:100])
    copes.cache_compact(cache)
    m.compact()
    follow()
    src, dst = list(range(0, 100)), list(range(300, 400))
    copes.cache_copy_pages(cache, ids(src), ids(dst))
    pool[300:400] = pool[0:100]
    assert error_bits(copes) == 0
    assert torch.equal(cache.pool.view(torch.int16), pool.view(torch.int16))


def test_a_fork_of_a_page_outside_the_pool_is_reported(copes):
    cache = copes.KVCache.empty(8, 1, 1, 4, 8, 3, 3)
    cache.pool.normal_()
    copes.cache_grow(cache, ids([0]), 6)
    cache.table[0, 1] = 77
    before = cache.pool.clone()
    copes.cache_fork(cache, ids([0, 0]), ids([1, 2]))
    assert error_bits(copes) == 32
    assert torch.equal(cache.pool, before)
    assert cache.table[1:, 0].tolist() == [0, 0] and cache.refs[0].item() == 3


def test_ids_outside_the_cache_are_skipped(copes):
    cache = copes.KVCache.empty(4, 1, 1, 4, 8, 2, 3)
    cache.pool.zero_()
    copes.cache_grow(cache, ids([0]), 6)
    k = torch.ones(1, 1, 8, device="cuda", dtype=torch.bfloat16)
    for slot, pos in ((2, 0), (-1, 0), (0, 6), (0, -1), (1, 0)):
        copes.cache_append(cache, 0, k, k, slots=ids([slot]), position=ids([pos]))
        assert error_bits(copes) == 32
    copes.cache_append(cache, 0, k.expand(2, 1, 8), k.expand(2, 1, 8))  # slot 1 has no last token
    assert error_bits(copes) == 32
    assert cache.pool.sum().item() == 16.0  # slot 0's last token alone, key and value
    copes.cache_copy_pages(cache, ids([0, 4, 0]), ids([-1, 1, 7]))
    assert error_bits(copes) == 32
    cache.table[0, 1] = 99
    copes.cache_append(cache, 0, k, k)
    assert error_bits(copes) == 32
    copes.cache_free(cache, ids([0]))
    assert error_bits(copes) == 32 and cache.refs[0].item() == 0
    assert error_bits(copes) == 0


# -------------------------------------------------------------------------- attention
def filled(copes, lens, layers, kv, page_size, d, dtype, seed, spare=3, poison=True):
    """A cache of sequences of these lengths on shuffled pages; what no token uses is NaN."""
    rng = np.random.default_rng(seed)
    pages = [-(-int(x) // page_size) for x in lens]
    n_pages = sum(pages) + spare
    order = rng.permutation(n_pages).astype(np.int32)
    width = max(max(pages), 1) + 1
    table = np.full((len(lens), width), -1, np.int32)
    refs = np.zeros(n_pages, np.int32)
    pool = torch.randn(n_pages, layers, 2, kv, page_size, d, device="cuda", generator=torch.Generator("cuda").manual_seed(seed))
    used = torch.zeros(n_pages, page_size, dtype=torch.bool)
    at = 0
    for i, p in enumerate(pages):
        table[i, :p] = order[at:at + p]
        refs[table[i, :p]] = 1
        for j in range(p):
            used[table[i, j], :min(page_size, int(lens[i]) - j * page_size)] = True
        at += p
    pool = pool.to(DT[dtype])
    if poison:
        pool.masked_fill_(~used.cuda()[:, None, None, None, :, None], float("nan"))
    t = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()
    return copes.KVCache(pool, t(table), t(lens), t(refs))


def check_attention(cache, layer, q, slots, scale, out, lse):
    """Against 64 bits.  With u the unit roundoff (2^-8 bf16, 2^-24 fp32): the output's rounding u |o|;
    a score's error, d + 4 roundings of at most 2^-24 S with S = sum |scale q k|, moves each weight
    twice (itself and the sum); weights rounded to two bf16 terms (2^-16), exp 2^-20, and sums of L
    terms 8 sqrt(L) 2^-24, all relative to sum p |v|."""
    ps, d = cache.desc.page_size, cache.desc.head_dim
    u = 2.0**-8 if q.dtype == torch.bfloat16 else 2.0**-24
    two_terms = 2.0**-16 if q.dtype == torch.bfloat16 else 0.0
    pool, table, length = f64(cache.pool[:, layer]), cache.table.cpu().numpy(), cache.length.cpu().numpy()
    qd, got, got_lse = f64(q), f64(out), f64(lse)
    worst = 0.0
    for i, s in enumerate(slots):
        n = int(length[s])
        rows = pool[table[s, :-(-n // ps)]] if n else np.zeros((0,) + pool.shape[1:])
        keys = rows[:, 0].transpose(0, 2, 1, 3).reshape(-1, pool.shape[2], d)[:n]
        vals = rows[:, 1].transpose(0, 2, 1, 3).reshape(-1, pool.shape[2], d)[:n]
        o, l, mass, size = model.attention(qd[i], keys, vals, scale)
        if n == 0:
            assert not got[i].any() and np.isneginf(got_lse[i]).all()
            continue
        score = (d + 4) * 2.0**-24 * size
        rel = 2 * score + two_terms + 2.0**-20 + 8 * np.sqrt(n) * 2.0**-24
        tol = 1.01 * u * np.abs(o) + rel[:, None] * mass + 1e-30
        assert np.isfinite(got[i]).all() and (np.abs(got[i] - o) <= tol).all(), (i, n, (np.abs(got[i] - o) / tol).max())
        worst = max(worst, (np.abs(got[i] - o) / tol).max())
        tol = score + 2.0**-20 + 8 * np.sqrt(n) * 2.0**-24 + 2.0**-23 * np.abs(l)
        assert (np.abs(got_lse[i] - l) <= tol).all(), (i, n)
    return worst


SHAPES = [  # q heads, kv heads, head_dim, page size
    (14, 2, 64, 16), (32, 8, 128, 16), (4, 4, 64, 1), (15, 5, 80, 7), (16, 1, 128, 64), (9, 1, 96, 50), (24, 3, 128, 33),
    (40, 1, 64, 16), (12, 4, 256, 16), (17, 1, 256, 8), (3, 3, 8, 5), (8, 2, 72, 128), (33, 1, 136, 16)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads,kv,d,ps", SHAPES)
def test_attention_matches_64_bits(copes, heads, kv, d, ps, dtype):
    lens = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 0, 300, 1000, 31, 777]
    cache = filled(copes, lens, 2, kv, ps, d, dtype, seed=heads + d)
    n = len(lens)
    qkv = (torch.randn(n, heads + 3, d + 5, device="cuda") * 1.5).to(DT[dtype])
    q = qkv[:, 2:2 + heads, :d]  # strides of rows and heads are not the shape's
    scale = d ** -0.5
    for layer in (0, 1):
        out, lse = copes.paged_attention(cache, layer, q)
        check_attention(cache, layer, q, range(n), scale, out, lse)
    slots = [13, 0, 14, 14, 3, 16]
    out, lse = copes.paged_attention(cache, 1, q[:6], slots=ids(slots), scale=0.3)
    check_attention(cache, 1, q[:6], slots, 0.3, out, lse)
    assert error_bits(copes) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,longest,heads,kv,d,ps", [(1, 20011, 32, 8, 128, 16), (1, 9001, 2, 1, 64, 16), (3, 7013, 14, 2, 64, 7),
                                                     (200, 90, 4, 2, 64, 16), (2, 4099, 12, 4, 256, 48),
                                                     (1000, 60, 4, 2, 64, 16), (420, 150, 12, 4, 128, 16), (500, 3000, 12, 4, 80, 16),
                                                     (470, 2000, 24, 8, 64, 7)])
def test_attention_split_over_long_and_many_sequences(copes, n, longest, heads, kv, d, ps, dtype):
    rng = np.random.default_rng(n)
    lens = rng.integers(0, min(longest, 200) + 1 if n > 100 else longest + 1, n)
    lens[-1] = longest
    cache = filled(copes, lens, 1, kv, ps, d, dtype, seed=n)
    q = (torch.randn(n, heads, d, device="cuda") * 3).to(DT[dtype])
    first = copes.paged_attention(cache, 0, q)
    check_attention(cache, 0, q, range(n), d ** -0.5, *first)
    for _ in range(3):  # joined in one order: the same bits again, on the same workspace
        again = copes.paged_attention(cache, 0, q)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    assert error_bits(copes) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_of_more_rows_than_a_block_keeps_lengths_of(copes, dtype):
    lens = np.random.default_rng(6).integers(0, 7, 9000)
    cache = filled(copes, lens, 1, 1, 4, 8, dtype, seed=6)
    q = torch.randn(9000, 2, 8, device="cuda").to(DT[dtype])
    out, lse = copes.paged_attention(cache, 0, q)
    check_attention(cache, 0, q, range(9000), 8 ** -0.5, out, lse)
    assert error_bits(copes) == 0


def test_attention_of_extreme_scores(copes):
    """One token outweighs all others by far, first or last; scores of +-1e4; equal scores."""
    for dtype in ("bf16", "fp32"):
        cache = filled(copes, [400, 400, 400, 400], 1, 1, 16, 64, dtype, seed=9)
        big = 100.0
        flat = cache.pool[:, 0, 0, 0]
        where = lambda i, t: (cache.table[i, t // 16].item(), t % 16)
        q = torch.ones(4, 4, 64, device="cuda", dtype=DT[dtype])
        flat[where(0, 0)] = big
        flat[where(1, 399)] = big
        for t in range(400):
            flat[where(2, t)] = -big if t != 200 else -big / 2
            flat[where(3, t)] = 1.0
        out, lse = copes.paged_attention(cache, 0, q, scale=1.0)
        check_attention(cache, 0, q, range(4), 1.0, out, lse)


@pytest.mark.parametrize("heads,kv,d,n", [(32, 8, 128, 128), (14, 2, 64, 700), (8, 4, 256, 16), (32, 2, 96, 32)])
def test_attention_of_long_rows_is_not_drawn_to_zero(copes, heads, kv, d, n):
    """Weighted means of 131,071 positive values, by rows on the same pages.  Rounding to bf16 is off by 2^-8 at
    most, either way, 2^-8 / sqrt(3) in the root mean square at most, independently for the kv d values: their mean
    error lies within six of its deviations.  (Sums that are cut 16,000 times by up to 2^-23 of them lose 2^-10.)"""
    tokens, pages = 131071, 8192
    generator = torch.Generator("cuda").manual_seed(d)
    pool = torch.rand(pages, 1, 2, kv, 16, d, device="cuda", generator=generator) + 0.5
    pool *= 2 ** torch.rand(kv, 1, d, device="cuda", generator=generator)
    pool = pool.bfloat16()
    table = torch.arange(pages, dtype=torch.int32, device="cuda").expand(n, pages).contiguous()
    cache = copes.KVCache(pool, table, ids([tokens] * n), ids([n] * pages))
    q = (torch.randn(d, device="cuda", generator=generator) * 0.3).bfloat16()
    out, lse = copes.paged_attention(cache, 0, q.expand(n, heads, d))
    keys, values = (pool[:, 0, i].transpose(0, 1).reshape(kv, -1, d)[:, :tokens].double() for i in (0, 1))
    scores = keys @ q.double() * d ** -0.5
    want = torch.einsum("gt,gtd->gd", torch.softmax(scores, -1), values)
    off = out.double().view(n, kv, heads // kv, d) / want[None, :, None] - 1
    assert off.abs().max() <= 1.01 * 2.0**-8
    assert off.mean().abs() <= 6 * 2.0**-8 / (3 * kv * d) ** 0.5
    assert (lse.double().view(n, kv, -1) - torch.logsumexp(scores, -1)[:, None]).abs().max() <= 2.0**-18
    assert error_bits(copes) == 0


def test_attention_of_the_largest_values(copes):
    """The largest fp32 values that a split leaves finite, as value, key and query, where the results are finite."""
    largest = [3.4019927e38, 3.4011621e38, 3.40039e38, 3.4e38]
    for d in (8, 72, 128, 256):
        cache = filled(copes, [1, 2, 1, 3], 1, 1, 4, d, "fp32", seed=d)
        cache.pool.nan_to_num_(0.0)
        page = lambda i: cache.pool[cache.table[i, 0].item(), 0, :, 0]  # [key or value][token][d]
        q = torch.zeros(4, 4, d, device="cuda")
        page(0)[1, 0] = torch.tensor([s * x for x in largest for s in (1, -1)], device="cuda").repeat(d // 8)
        page(1)[1, 0], page(1)[1, 1] = largest[0], -largest[0]
        page(2)[0, 0, 0] = -largest[0]  # a score of -2.6 by a tiny query and this scale
        q[2, :, 0] = 2.0**-120
        page(3)[0, :3, 1] = torch.tensor([2.0**-124, -2.0**-123, 2.0**-122], device="cuda")
        q[3, :, 1] = torch.tensor(largest, device="cuda")
        out, lse = copes.paged_attention(cache, 0, q, scale=0.01)
        check_attention(cache, 0, q, range(4), 0.01, out, lse)


def test_attention_reports_ids_outside_the_cache(copes):
    cache = filled(copes, [20, 40], 1, 2, 16, 64, "bf16", seed=3)
    q = torch.randn(3, 4, 64, device="cuda").bfloat16()
    out, lse = copes.paged_attention(cache, 0, q, slots=ids([2, 1, -5]))
    assert error_bits(copes) == 32
    assert not out[[0, 2]].any() and torch.isneginf(lse[[0, 2]]).all()
    check_attention(cache, 0, q[1:2], [1], 64 ** -0.5, out[1:2], lse[1:2])
    cache.table[1, 1] = 1 << 30
    cache.table[0, 0] = -7
    out, lse = copes.paged_attention(cache, 0, q[:2])
    assert error_bits(copes) == 32 and torch.isfinite(out).all()
    cache.length[0] = -3  # a length that no call writes
    cache.length[1] = 1 << 30
    cache.table.fill_(0)
    out, lse = copes.paged_attention(cache, 0, q[:2])
    assert error_bits(copes) == 0 and not out[0].any()


def test_attention_past_32_bits(copes):
    """Pages whose elements start past 2^32 of the pool."""
    n_pages = (1 << 32) // (2 * 2 * 16 * 128) + 40
    pool = torch.empty(n_pages, 1, 2, 2, 16, 128, device="cuda", dtype=torch.bfloat16)
    cache = copes.KVCache(pool, torch.full((1, 8), -1, dtype=torch.int32, device="cuda"), ids([0]),
                          torch.zeros(n_pages, dtype=torch.int32, device="cuda"))
    cache.refs[:n_pages - 5] = 1
    copes.cache_grow(cache, ids([0]), 70)
    assert cache.table[0, :6].tolist() == [n_pages - 5, n_pages - 4, n_pages - 3, n_pages - 2, n_pages - 1, -1]
    kv = torch.randn(70, 2, 2, 128, device="cuda").bfloat16()
    copes.cache_append(cache, 0, kv[:, 0], kv[:, 1], slots=ids([0] * 70), position=ids(range(70)))
    q = torch.randn(1, 8, 128, device="cuda").bfloat16()
    out, lse = copes.paged_attention(cache, 0, q)
    small = copes.KVCache(pool[-5:].clone(), ids([0, 1, 2, 3, 4])[None].contiguous(), ids([70]), ids([1] * 5))
    check_attention(small, 0, q, [0], 128 ** -0.5, out, lse)
    cache.refs[:n_pages - 5] = 0
    copes.cache_compact(cache)
    assert cache.table[0, :5].tolist() == [0, 1, 2, 3, 4]
    again = copes.paged_attention(cache, 0, q)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    assert error_bits(copes) == 0


def test_calls_run_on_the_stream_they_are_given_and_in_a_graph(copes):
    cache = filled(copes, [500, 33, 0], 1, 2, 16, 64, "bf16", seed=4)
    q = torch.randn(3, 14, 64, device="cuda").bfloat16()
    want = copes.paged_attention(cache, 0, q)
    logits = torch.randn(3, 5000, device="cuda").bfloat16()
    target = torch.tensor([1, 2, 3], device="cuda")
    want_lp = copes.token_logprobs(logits, target, top=4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = copes.paged_attention(cache, 0, q, stream=side)
    got_lp = copes.token_logprobs(logits, target, top=4, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(got_lp.logprob, want_lp.logprob) and torch.equal(got_lp.top_ids, want_lp.top_ids)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = copes.paged_attention(cache, 0, q)
        held_lp = copes.token_logprobs(logits, target, top=4)
    for _ in range(2):
        held[0].zero_()
        held_lp.logprob.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held[0], want[0]) and torch.equal(held[1], want[1])
        assert torch.equal(held_lp.logprob, want_lp.logprob) and torch.equal(held_lp.entropy, want_lp.entropy)
    assert error_bits(copes) == 0


def test_cache_calls_in_a_graph(copes):
    """Replays of a captured step do what the calls do one after the other: every page, count and value."""
    d, kv, layers, ps = 64, 2, 3, 4
    k, v = torch.randn(2, 3, kv, d, device="cuda").bfloat16()
    rows, child, counts = ids([0, 1, 2]), ids([3, 4]), ids([0, 0])
    src, dst = ids([2, 5]), ids([38, 39])

    def fresh():
        cache = copes.KVCache.empty(40, layers, kv, ps, d, 5, 6)
        cache.pool.copy_(torch.arange(cache.pool.numel(), device="cuda").view(cache.pool.shape) % 251)
        copes.cache_grow(cache, rows, ids([3, 9, 0]))
        copes.cache_append(cache, 1, k, v, slots=ids([0, 1, 1]), position=ids([1, 8, 0]))
        copes.cache_free(cache, ids([0]))
        copes.cache_grow(cache, ids([0]), 2)
        return cache

    def step(cache):
        copes.cache_grow(cache, rows, 1)
        copes.cache_append(cache, 2, k, v, slots=rows)
        copes.cache_fork(cache, rows[1:], child)
        copes.cache_copy_pages(cache, src, dst)
        copes.cache_free(cache, rows[1:2])
        copes.cache_compact(cache, counts)
        copes.cache_free(cache, child)
        copes.cache_grow(cache, rows[1:2], 5)

    cache, want = fresh(), fresh()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cache)
    for _ in range(8):
        graph.replay()
        got = counts.clone()
        step(want)
        assert error_bits(copes) == 0
        assert torch.equal(got, counts) and torch.equal(cache.pool, want.pool)
        for name in ("table", "length", "refs"):
            assert torch.equal(getattr(cache, name), getattr(want, name)), name


def test_a_graph_keeps_the_workspace_it_was_captured_with(copes):
    """A larger call between capture and replay: the graph's workspace is nobody else's then."""
    lens = [3000] + [40] * 299
    cache = filled(copes, lens, 1, 2, 16, 64, "bf16", seed=11)
    q = torch.randn(300, 14, 64, device="cuda").bfloat16()
    want = copes.paged_attention(cache, 0, q[:1])
    captured = cache.attend_workspace.data_ptr(), cache.attend_workspace.numel()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = copes.paged_attention(cache, 0, q[:1])
    copes.paged_attention(cache, 0, q)
    assert cache.attend_workspace.data_ptr() != captured[0]  # the call was large enough to need more
    others = [torch.full((captured[1],), 7, dtype=torch.uint8, device="cuda") for _ in range(8)]
    assert all(x.data_ptr() != captured[0] for x in others)
    for x in held:
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(held[0], want[0]) and torch.equal(held[1], want[1])
    assert all((x == 7).all() for x in others)
    assert error_bits(copes) == 0


def test_a_dropped_handle_keeps_its_memory_until_its_streams_are_through(copes):
    cache = filled(copes, [2000, 33, 700], 1, 2, 16, 64, "bf16", seed=12)
    q = torch.randn(3, 14, 64, device="cuda").bfloat16()
    want = copes.paged_attention(cache, 0, q)
    arrays = (cache.pool, cache.table, cache.length, cache.refs, cache.workspace, cache.attend_workspace)
    held = [(t.data_ptr(), t.numel() * t.element_size()) for t in arrays]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)  # cycles: some 50 ms
    out, lse = copes.paged_attention(cache, 0, q, stream=side)
    del cache, arrays
    others = [torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda") for _, size in held for _ in range(3)]
    busy = not side.query()
    for x in others:
        assert all(x.data_ptr() + x.numel() <= at or at + size <= x.data_ptr() for at, size in held)
    assert busy  # else the check above says nothing
    side.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert error_bits(copes) == 0


# ---------------------------------------------------------------- token log probabilities
def check_logprobs(copes, logits, target, top, scale=1.0):
    """ids exactly.  Numbers: the subtraction from the maximum, the product with the scale and the
    final difference round to 2^-24 of their sizes; the sum of V positive terms of relative error
    2^-20 adds 2^-20 + V / 128 roundings of 2^-24 (no sum here is longer); the entropy's terms are
    off by that relative to |p ln p|."""
    r = copes.token_logprobs(logits, target, top=top, scale=scale)
    assert error_bits(copes) == (32 if (target >= logits.shape[1]).any() else 0)
    x, t = f64(logits), target.cpu().numpy()
    scale = float(np.float32(scale))
    lp, en, tid, tlp = f64(r.logprob), f64(r.entropy), r.top_ids.cpu().numpy(), f64(r.top_logprobs)
    part = 2.0**-20 + max(1, x.shape[1] / 128) * 2.0**-24
    for i in range(x.shape[0]):
        a, e, wid, wlp, lse = model.token_logprobs(x[i], int(t[i]), top, scale)
        assert np.array_equal(tid[i], wid), i
        for got, want in [(lp[i], a)] + list(zip(tlp[i], wlp)):
            with np.errstate(over="ignore"):  # a value past fp32 is infinite
                want = want if abs(want) <= np.finfo(np.float32).max else np.float64(np.float32(want))
            if not np.isfinite(want):
                assert np.array_equal(got, want, equal_nan=True), (i, got, want)
                continue
            assert abs(got - want) <= part + 2.0**-22 * (abs(want) + 1), (i, got, want)
        if np.isnan(e):
            assert np.isnan(en[i])
        else:
            assert abs(en[i] - e) <= 4 * part * (1 + e) + 2.0**-22 * 8, (i, en[i], e)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,vocab,top", [(1, 1, 1), (2, 2, 2), (3, 7, 7), (5, 31, 3), (4, 32, 32), (3, 255, 5), (2, 257, 32), (3, 512, 1),
                                         (2, 513, 20), (7, 4095, 8), (1, 32003, 20), (33, 32003, 0), (1, 151936, 32),
                                         (3, 151936, 20), (40, 151936, 5), (170, 10007, 3), (700, 1031, 4)])
def test_logprobs_match_64_bits(copes, n, vocab, top, dtype):
    g = torch.Generator("cuda").manual_seed(vocab + n)
    wide = (torch.randn(n, vocab + 3, device="cuda", generator=g) * 3).to(DT[dtype])
    target = torch.randint(0, vocab, (n,), device="cuda", generator=g)
    target[n // 2] = -1 if n > 2 else target[n // 2]
    check_logprobs(copes, wide[:, :vocab].contiguous(), target, top)
    check_logprobs(copes, wide[:, 1:1 + vocab], target, top, scale=1.43)  # rows that start anywhere


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [5, 300, 3001, 70001])
def test_logprobs_of_ties_masks_and_orders(copes, vocab, dtype):
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
    rows = [up, up.flip(0), torch.full((vocab,), 1.5, device="cuda"), torch.full((vocab,), -torch.inf, device="cuda"), few, last,
            zeros, block, lows, torch.full((vocab,), low, device="cuda"), torch.full((vocab,), -low, device="cuda"),
            torch.randint(0, 3, (vocab,), device="cuda", generator=g).float(),
            torch.where(torch.rand(vocab, device="cuda", generator=g) < 0.9, -torch.inf, up)]
    nan = up.clone()
    nan[vocab // 2] = torch.nan
    nan[0] = -torch.nan
    inf = up.clone()
    inf[1] = torch.inf
    both = inf.clone()
    both[vocab - 1] = torch.nan
    rows += [nan, inf, both, torch.full((vocab,), torch.nan, device="cuda")]
    logits = torch.stack(rows).to(DT[dtype])
    n = len(rows)
    for target in (torch.full((n,), vocab - 1, device="cuda"), torch.zeros(n, dtype=torch.int64, device="cuda"),
                   torch.full((n,), -7, device="cuda"), torch.full((n,), vocab, device="cuda")):
        for top in (0, 1, min(vocab, 20), min(vocab, 32)):
            check_logprobs(copes, logits, target, top)
    check_logprobs(copes, logits[:1], target[:1] * 0, min(vocab, 5), scale=0.01)
    check_logprobs(copes, logits, target * 0, min(vocab, 5), scale=3.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,vocab", [(1, 151936), (400, 20011), (1, 700001)])
def test_logprobs_whose_largest_recur(copes, n, vocab, dtype):
    """The largest logits in one 16-byte piece of every 32: most threads see none of them, so hundreds surpass what
    is known of the alternatives when the row has been read."""
    piece = 8 if dtype == "bf16" else 4
    g = torch.Generator("cuda").manual_seed(vocab)
    logits = torch.randn(n, vocab, device="cuda", generator=g).to(DT[dtype])
    place = torch.arange(vocab, device="cuda")
    large = place // piece % 32 == 7
    logits[:, large] = (torch.randn(n, int(large.sum()), device="cuda", generator=g) + 20).to(DT[dtype])
    target = torch.randint(0, vocab, (n,), device="cuda", generator=g)
    for top in (5, 32):
        check_logprobs(copes, logits, target, top)


def test_logprobs_rows_past_32_bits(copes):
    """Rows whose elements start past 2^32."""
    row = 1 << 31
    logits = torch.empty(2 * row + 400, device="cuda", dtype=torch.bfloat16).as_strided((3, 400), (row, 1))
    logits.copy_(torch.randn(3, 400, device="cuda"))
    check_logprobs(copes, logits, torch.tensor([5, 399, 0], device="cuda"), 10)
