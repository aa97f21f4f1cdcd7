"""Calls at the edges of a generating step that the host decides: pools of another form, weights of another type than
the cache, cuts that fp32 rounds away, and what a decoder leaves in a cache where a step fails."""
import glob
import os
import re
from types import SimpleNamespace

import pytest
import torch


@pytest.fixture(scope="module")
def copes():
    from paper_2608_02391_gb300 import build, copes as c
    if not os.path.exists(c.LIB_PATH):
        build.build()
    c.load()
    return c


class OnGpu:
    """A tensor on a GPU, as far as a cache's handle looks at it."""
    is_cuda, device = True, torch.device("cpu")

    def __init__(self, at, dtype, *shape):
        self.at, self.dtype, self.shape = at, dtype, torch.Size(shape)

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.at


def handle(copes, pool, **kw):
    i32 = torch.int32
    return copes.KVCache(pool, OnGpu(0x9000000, i32, 3, 4), OnGpu(0xA000000, i32, 3), OnGpu(0xB000000, i32, pool.shape[0]), **kw)


def test_bytes_are_a_pool_only_with_room_for_their_exponents(copes, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: type("Stream", (), {"cuda_stream": 0}))
    for dtype in (torch.uint8, torch.int8, torch.float16, torch.float8_e4m3fn):
        for page_size, d in ((16, 16), (1, 256), (64, 64)):
            with pytest.raises(KeyError):
                handle(copes, OnGpu(0x1000000, dtype, 4, 1, 2, 1, page_size, d))
    for dtype, code in ((torch.bfloat16, copes.BF16), (torch.float32, copes.FP32)):
        c = handle(copes, OnGpu(0x1000000, dtype, 4, 1, 2, 1, 16, 16))
        assert (c.dtype, c.io_dtype, c.heads) == (code, dtype, (1, 16, 16))
    room = copes.KVCache.layer_bytes(1, 16, 16)
    c = handle(copes, OnGpu(0x1000000, torch.uint8, 4, 1, room), heads=(1, 16, 16))
    assert (c.dtype, c.io_dtype, c.heads) == (copes.E4M3, torch.bfloat16, (1, 16, 16))
    for n in (room - 16, 2 * 16 * 16, room + 16):
        with pytest.raises(AssertionError):
            handle(copes, OnGpu(0x1000000, torch.uint8, 4, 1, n), heads=(1, 16, 16))


def test_cluster_barriers_take_lanes_one_by_one():
    """barrier.cluster with .aligned is undefined where a warp's lanes are not together, and lanes come to the kernels' barriers
    from loops and branches of their own.  Which barrier a kernel asks for is in its source alone."""
    root = os.path.join(os.path.dirname(__file__), "..", "paper_2608_02391_gb300", "csrc")
    asked = [b for f in glob.glob(os.path.join(root, "*.cu*")) + glob.glob(os.path.join(root, "*.h"))
             for b in re.findall(r"barrier\.cluster\.(?:arrive|wait)[.a-z]*", open(f).read())]
    assert len(asked) >= 4 and not [b for b in asked if "aligned" in b]


SHAPE = dict(layers=2, hidden=48, mlp=80, vocab=301, q_heads=6, kv_heads=2, head_dim=16)


def decoder_and_weights(dtype, **kw):
    from paper_2608_02391_gb300 import rollout
    d = rollout.Decoder(rollout.Shape(**{**SHAPE, **kw}), device="cpu")
    return d, torch.zeros(d.offsets[-1] + d.tensors[-1].numel, dtype=dtype)


def cache_of(copes, dtype, heads=(2, 16, 16), layers=2):
    code, io = (copes.E4M3, torch.bfloat16) if dtype is None else (copes._DTYPE_CODES[dtype], dtype)
    return SimpleNamespace(desc=copes.KVCacheDesc(1, code, 100, layers, *heads, 1, 9, 9, 1, 1), pool=torch.zeros(1), heads=heads, io_dtype=io,
                           length=torch.zeros(9, dtype=torch.int32), refs=torch.zeros(100, dtype=torch.int32))


def calls_of(d, w, cache):
    prompts, u = [[1, 2], [3]], torch.zeros(3, 4)
    return [lambda: d.score(w, cache, prompts, [[[1]], [[2, 3]]]), lambda: d.greedy(w, cache, prompts, 3),
            lambda: d.sample(w, cache, prompts, 3, u[:, :2]), lambda: d.sample(w, cache, prompts, 3, u, rollouts=2),
            lambda: d.read(d.weights(w), cache, [0, 1], prompts)]


class Begun(Exception):
    pass


def test_caches_of_other_weights_are_refused_before_any_work(copes, monkeypatch):
    """None: a cache in 8 bits, for bf16."""
    def begun(*a, **kw):
        raise Begun

    monkeypatch.setattr(copes, "cache_grow", begun)
    monkeypatch.setattr(copes, "cache_free", lambda *a, **kw: None)
    bf16, fp32 = torch.bfloat16, torch.float32
    for weights, cache, fine in ((fp32, None, False), (fp32, bf16, False), (bf16, fp32, False), (bf16, None, True), (bf16, bf16, True),
                                 (fp32, fp32, True)):
        for call in calls_of(*decoder_and_weights(weights), cache_of(copes, cache)):
            with pytest.raises(Begun if fine else ValueError, match=None if fine else "cache"):
                call()
    for kw in (dict(heads=(4, 16, 16)), dict(heads=(2, 16, 32)), dict(layers=1)):
        for call in calls_of(*decoder_and_weights(bf16), cache_of(copes, bf16, **kw)):
            with pytest.raises(ValueError, match="cache"):
                call()
    for call in calls_of(*decoder_and_weights(bf16), cache_of(copes, bf16, layers=3)):
        with pytest.raises(Begun):
            call()


def test_cuts_that_fp32_rounds_away_are_refused_before_any_work(copes, monkeypatch):
    def begun(*a, **kw):
        raise Begun

    monkeypatch.setattr(copes, "cache_grow", begun)
    monkeypatch.setattr(copes, "cache_free", lambda *a, **kw: None)
    d, w = decoder_and_weights(torch.bfloat16)
    for kw, fine in ((dict(top_p=1e-46), False), (dict(top_p=5e-324), False), (dict(top_p=2e-45), True), (dict(min_p=1e-46), True),
                     (dict(top_p=1 - 1e-12), True), (dict(temperature=1e-38), True), (dict(temperature=1e30), True)):
        with pytest.raises(Begun if fine else ValueError, match=None if fine else "cuts"):
            d.sample(w, cache_of(copes, torch.bfloat16), [[1, 2]], 3, torch.zeros(3, 1), **kw)


@pytest.mark.parametrize("fails", ["read", "step", "cache_fork"])
def test_slots_are_empty_after_work_that_fails(copes, monkeypatch, fails):
    """Each call frees the slots that it was to use, once, whether reading, forking or a later step fails."""
    def failing(*a, **kw):
        raise Begun

    freed = []
    monkeypatch.setattr(copes, "cache_free", lambda cache, slots, **kw: freed.append(slots.tolist()))
    monkeypatch.setattr(copes, "cache_fork", failing if fails == "cache_fork" else lambda *a, **kw: None)
    ones = lambda logits, *a, **kw: SimpleNamespace(logprob=torch.zeros(len(logits)), top_ids=torch.zeros(len(logits), 1, dtype=torch.int64),
                                                    ids=torch.zeros(len(logits), dtype=torch.int64))
    monkeypatch.setattr(copes, "token_logprobs", ones)
    monkeypatch.setattr(copes, "sample_tokens", ones)
    d, w = decoder_and_weights(torch.bfloat16)
    monkeypatch.setattr(d, "read", failing if fails == "read" else lambda weights, cache, slots, prompts: torch.zeros(len(prompts), 301))
    monkeypatch.setattr(d, "step", failing)
    prompts, u, cache = [[1, 2], [3]], torch.zeros(3, 4), cache_of(copes, torch.bfloat16)
    for n, call in ((5, lambda: d.score(w, cache, prompts, [[[1]], [[2, 3], [4, 5, 6]]])), (2, lambda: d.greedy(w, cache, prompts, 3)),
                    (2, lambda: d.sample(w, cache, prompts, 3, u[:, :2])), (6, lambda: d.sample(w, cache, prompts, 3, u, rollouts=2))):
        if fails == "cache_fork" and n == 2:
            continue
        freed.clear()
        with pytest.raises(Begun):
            call()
        assert freed == [list(range(n))]


def test_a_decoder_without_layers_takes_any_cache(copes, monkeypatch):
    """It writes nothing there."""
    for name in ("cache_grow", "cache_free"):
        monkeypatch.setattr(copes, name, lambda *a, **kw: None)
    d, w = decoder_and_weights(torch.float32, layers=0)
    logits = d.read(d.weights(w), cache_of(copes, torch.bfloat16, heads=(1, 16, 64), layers=1), [0, 1], [[1, 2], [3]])
    assert logits.shape == (2, 301)
