"""A generating step's calls at the edges of what they allow: heads of a page past 2^31 tokens."""
import numpy as np
import pytest
import torch

import step_model as model

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
