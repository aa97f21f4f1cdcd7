"""What drawing rollouts refuses before any work, and what a decoder's norms add up to on the CPU."""
import random
from types import SimpleNamespace

import pytest
import torch

import answer_model as model
from paper_2608_02391_gb300 import copes, rollout, workloads

SHAPE = rollout.Shape(2, 48, 80, 301, q_heads=6, kv_heads=2, head_dim=16)


def cache_of(n_pages, page_size, n_slots, width):
    return SimpleNamespace(desc=copes.KVCacheDesc(1, 0, n_pages, 2, 2, page_size, 16, 1, n_slots, width, 1, 1), pool=torch.zeros(1),
                           length=torch.zeros(n_slots, dtype=torch.int32), refs=torch.zeros(n_pages, dtype=torch.int32))


def draw(cache, prompts, n_tokens, u=None, rollouts=1, **kw):
    u = torch.zeros(max(n_tokens, 0), max(len(prompts) * rollouts, 0)) if u is None else u
    return rollout.Decoder(SHAPE, device="cpu").sample(None, cache, prompts, n_tokens, u, rollouts=rollouts, **kw)


def refused(match, *args, **kw):
    with pytest.raises(ValueError, match=match):
        draw(*args, **kw)


def test_rollouts_that_are_refused():
    cache = cache_of(100, 16, 9, 9)
    refused("no prompts", cache, [], 3)
    refused("empty prompt", cache, [[1], []], 3)
    refused("vocabulary", cache, [[1], [301]], 3)
    for n_tokens, rollouts in ((0, 1), (-1, 2), (3, 0), (3, -2)):
        refused("continuations", cache, [[1]], n_tokens, u=torch.zeros(3, 1), rollouts=rollouts)
    for temperature in (0.0, -1.0, float("nan"), float("inf"), 1e-39):
        refused("temperature", cache, [[1]], 3, temperature=temperature)
    for kw in (dict(top_k=-1), dict(top_p=0.0), dict(top_p=1.5), dict(top_p=float("nan")), dict(min_p=-0.1), dict(min_p=2.0)):
        refused("cuts", cache, [[1]], 3, **kw)
    refused("random numbers", cache, [[1], [2]], 3, u=torch.zeros(3, 3))
    refused("random numbers", cache, [[1], [2]], 3, u=torch.zeros(2, 2))
    refused("random numbers", cache, [[1], [2]], 3, u=torch.zeros(3, 2, dtype=torch.float64))
    refused("slots", cache_of(100, 16, 8, 9), [[1], [2], [3]], 3, rollouts=2)
    refused("slots", cache_of(100, 16, 2, 9), [[1], [2], [3]], 3)
    refused("tokens", cache_of(100, 4, 9, 3), [[1] * 10], 4)
    busy = cache_of(100, 16, 9, 9)
    busy.length[2] = 1
    refused("not empty", busy, [[1]], 3, rollouts=2)


def test_pages_that_rollouts_need_are_those_they_take():
    """Against the pages in use when all is written, by the model of the bookkeeping: with so many the room is
    there (and the next thing that is asked for is weights), with one less it is not."""
    rng = random.Random(9)
    for _ in range(200):
        size, rollouts, n_tokens = rng.choice([1, 3, 7, 16]), rng.choice([1, 1, 2, 5]), rng.randint(1, 30)
        prompts = [[1] * rng.randint(1, 40) for _ in range(rng.randint(1, 4))]
        first = len(prompts)
        n = first + (first * rollouts if rollouts > 1 else 0)
        m = model.CacheModel(4000, size, n, 100)
        assert m.grow(range(first), [len(p) for p in prompts]) == 0
        if rollouts == 1:
            assert m.grow(range(first), [n_tokens - 1] * first) == 0
        else:
            children = list(range(first, n))
            assert m.fork([i for i in range(first) for _ in range(rollouts)], children) == 0
            assert m.grow(children, [n_tokens - 1] * len(children)) == 0
        need, longest = sum(r != 0 for r in m.refs), max(m.length)
        with pytest.raises(TypeError):  # past the checks: there are no weights
            draw(cache_of(need, size, n, -(-longest // size)), prompts, n_tokens, rollouts=rollouts)
        for few in ((need - 1, size, n, 100), (need, size, n - 1, 100)):
            if few[0] and few[2]:
                with pytest.raises(ValueError):
                    draw(cache_of(*few), prompts, n_tokens, rollouts=rollouts)


def test_layouts_without_the_new_tensors_are_as_they_were():
    old = [(t.name, t.numel, t.kind) for t in workloads.decoder_tensors(2, 48, 80, 301, 6, 2, 16, True, True, False)]
    new = [(t.name, t.numel, t.kind) for t in rollout.Shape(2, 48, 80, 301, 6, 2, 16, True, True, False, out_norms=True,
                                                            block_gates=True).tensors()]
    assert [t for t in new if not t[0].startswith(("l0.attn_", "l1.attn_", "l0.mlp_", "l1.mlp_"))] == old and len(new) == len(old) + 8
    assert rollout.Decoder(SHAPE, device="cpu").fused is False
    for kw in (dict(out_norms=True), dict(block_gates=True), dict(residual_scale=0.5)):
        assert rollout.Decoder(rollout.Shape(2, 48, 80, 301, 6, 2, 16, **kw), device="cpu").fused
