"""A generating step's calls at the edges of what they allow: heads of a page past 2^31 tokens, queries and keys of any size,
norms whose eps counts beside squares past fp32."""
import numpy as np
import pytest
import torch

import step_model as model
from test_gpu_step import cache8, check_attention, check_norm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def copes():
    from paper_2608_02391_gb300 import copes as c
    c.load()
    return c


def ids(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def f64(t):
    return t.detach().double().cpu().numpy()


def test_heads_of_a_page_past_2_to_31_tokens(copes):
    """33 heads of 2^26 tokens in one page of an 8-bit cache: the last head's bytes begin past 2^31 of them (75 GB, of which a few are
    written).  Against a cache of small pages with the same tokens."""
    kv, ps, d, n = 33, 1 << 26, 16, 5
    if torch.cuda.mem_get_info()[0] < 1.1 * copes.KVCache.layer_bytes(kv, ps, d):
        pytest.skip("less than 83 GB free")
    kv_rows = torch.randn(n, 2, kv, d, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    kv_rows = (kv_rows * 2.0 ** torch.arange(-16, 17, device="cuda")[:, None]).bfloat16()  # each head with another byte
    q, got, cache = torch.randn(1, kv, d, device="cuda").bfloat16(), [], None
    try:
        for page_size in (ps, 16):
            cache = copes.KVCache.empty(1, 1, kv, page_size, d, 1, 1, dtype=torch.float8_e4m3fn)
            copes.cache_grow(cache, ids([0]), n)
            slots, position = ids([0] * n), ids(range(n))
            copes.cache_append(cache, 0, kv_rows[:, 0], kv_rows[:, 1], slots=slots, position=position)
            read = copes.cache_read(cache, 0, slots=slots, position=position)
            for x, want in zip(read, (kv_rows[:, 0], kv_rows[:, 1])):
                assert np.array_equal(f64(x), model.stored(f64(want))[0])
            got.append(copes.paged_attention(cache, 0, q, scale=2.0**-20))
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
        copes.check()
    finally:
        cache = None
        torch.cuda.empty_cache()


# log2 of the queries, of the keys' powers of two, of the scale: scores of some units each
SIZES = [(0, -3, -9), (60, -66, -6), (120, -120, -12), (110, -113, -9), (100, -100, -12), (-110, 100, -2), (-125, 118, -5), (-129, 118, -1),
         (-121, -1, 110), (-128, 0, 116), (60, 50, -122), (-60, -50, 98)]


@pytest.mark.parametrize("heads,kv,d", [(6, 2, 64), (32, 2, 64), (12, 4, 128), (10, 5, 256)])
@pytest.mark.parametrize("query,key,scale", SIZES)
def test_queries_and_keys_of_any_size(copes, query, key, scale, heads, kv, d):
    """Products of queries and keys that fp32 holds, of factors that are as large and as small as their types hold: a query's
    values of at least 2^-32 of its largest count whole, in bf16's subnormal numbers, too."""
    ps, lens = 16, [1, 16, 40, 333, 0, 700]
    cache = cache8(copes, lens, 1, kv, ps, d, seed=d + heads)
    size, rng = 2 * kv * ps * d, np.random.default_rng(heads)
    powers = rng.integers(116, 122, (cache.desc.n_pages, 1, 2, kv, ps))
    powers[:, :, 0] = key + 127 - rng.integers(0, 6, powers[:, :, 0].shape)
    powers = np.maximum(powers, 1)
    cache.pool[:, :, size:size + 2 * kv * ps] = torch.from_numpy(powers.reshape(cache.desc.n_pages, 1, -1).astype(np.uint8)).cuda()
    g = torch.Generator("cuda").manual_seed(heads)
    q = (torch.randn(len(lens), heads, d, device="cuda", generator=g, dtype=torch.float64) * 2.0**query).bfloat16()
    q[:, 0] = 0
    q[:, 1, 5:] = (q[:, 1, 5:].double() * 2.0**-20).bfloat16()
    q[1, 2:4] = (q[1, 2:4].double() * 2.0**-30).bfloat16()  # beside others of its kind
    scale = 2.0**scale
    check_attention(cache, 0, q, range(len(lens)), scale, *copes.paged_attention(cache, 0, q, scale=scale))
    copes.check()


@pytest.mark.parametrize("n,hidden", [(3, 64), (2, 4096), (2500, 4096), (2, 8192), (2, 8190), (2, 300_000), (2, 1 << 24)])
def test_eps_counts_beside_squares_past_fp32(copes, n, hidden):
    """Squares whose sum is just past fp32, so that their mean is 2e31 and more, and the largest eps, 1e30."""
    eps = 1e30
    sign = torch.randint(0, 2, (n, hidden), device="cuda", generator=torch.Generator("cuda").manual_seed(hidden)).float() * 2 - 1
    x = sign * (1.02 * (torch.finfo(torch.float32).max / hidden) ** 0.5)
    x[n // 2] *= 0.5  # its sum is not
    w = torch.linspace(0.5, 1.5, hidden, device="cuda")
    rows = torch.tensor(sorted({0, n // 2, n - 1} | set(range(0, n, 200))), device="cuda")
    _, h = copes.residual_norm(x, w, eps=eps)
    check_norm(None, h[rows], x[rows], w, None, None, None, 1.0, eps)
    zeros = torch.zeros_like(x)
    s, h = copes.residual_norm(zeros, w, y=x, out_weight=w, scale=0.5, eps=eps)
    check_norm(s[rows], h[rows], zeros[rows], w, x[rows], w, None, 0.5, eps)
    s, h = copes.residual_norm(zeros, w, y=x, eps=eps)
    check_norm(s[rows], h[rows], zeros[rows], w, x[rows], None, None, 1.0, eps)
    copes.check()
