"""What a decoder refuses before any work: every case is decided by the host, on a cache that has a
cache's sizes and counts and nothing else."""
import random
from types import SimpleNamespace

import pytest
import torch

import answer_model as model
from paper_2608_02391_gb300 import copes, rollout

SHAPE = rollout.Shape(2, 48, 80, 301, q_heads=6, kv_heads=2, head_dim=16)


def cache_of(n_pages, page_size, n_slots, width):
    return SimpleNamespace(desc=copes.KVCacheDesc(1, 0, n_pages, 2, 2, page_size, 16, 1, n_slots, width, 1, 1),
                           length=torch.zeros(n_slots, dtype=torch.int32), refs=torch.zeros(n_pages, dtype=torch.int32))


def refused(match, cache, prompts, answers, n_tokens=4):
    """By score and by greedy; None for the one that is not asked."""
    d = rollout.Decoder(SHAPE, device="cpu")
    if answers is not None:
        with pytest.raises(ValueError, match=match):
            d.score(None, cache, prompts, answers)
    if n_tokens is not None:
        with pytest.raises(ValueError, match=match):
            d.greedy(None, cache, prompts, n_tokens)


def test_work_that_the_cache_has_no_room_for_is_refused():
    prompts, answers = [[1] * 5, [2] * 16], [[[3] * 4, [4]], [[5] * 17]]
    refused("slots", cache_of(100, 16, 4, 9), prompts, answers, None)
    refused("slots", cache_of(100, 16, 1, 9), prompts, None)
    refused("slots", cache_of(100, 16, 64, 9), [[1]] * 40, [[[1]]] * 40, None)
    refused("tokens", cache_of(100, 4, 5, 7), prompts, answers, None)  # 32 tokens
    refused("tokens", cache_of(100, 3, 5, 6), prompts, None)           # 19 tokens
    refused("tokens", cache_of(100, 5, 5, 3), [[1] * 16], [[[1]]], 1)
    busy = cache_of(100, 16, 5, 9)
    busy.length[1] = 1
    refused("not empty", busy, prompts, answers)
    full = cache_of(5, 16, 5, 9)
    full.refs[3] = 1  # of the 5 that are needed: two for the prompts, and one for each answer's own tokens
    refused("pages", full, prompts, answers, None)
    refused("pages", cache_of(2, 16, 5, 9), prompts, None)  # 8 and 19 tokens


def test_sequences_without_tokens_are_refused():
    cache = cache_of(100, 16, 9, 9)
    refused("empty answer", cache, [[1], [2]], [[[3], []], [[4]]], None)
    refused("empty prompt", cache, [[1], []], [[[3]], [[4]]])
    refused("no answers", cache, [[1], [2]], [[], []], None)
    refused("no answers", cache, [[1], [2]], [], None)
    refused("no prompts", cache, [], [])
    for n_tokens in (0, -1):
        refused("continuation", cache, [[1]], None, n_tokens)
    d = rollout.Decoder(SHAPE, device="cpu")
    for prompts in ([], [[1], []]):
        with pytest.raises(ValueError):
            d.read({}, cache, [0, 1], prompts)


def test_tokens_outside_the_vocabulary_and_answers_without_a_prompt_are_refused():
    cache = cache_of(100, 16, 9, 9)
    for bad in (301, -1, 2**40, -301):
        refused("vocabulary", cache, [[1], [2, bad]], [[[3]], [[4]]])
        refused("vocabulary", cache, [[1], [2]], [[[3]], [[4, 0], [0, bad]]], None)
        with pytest.raises(ValueError):
            rollout.Decoder(SHAPE, device="cpu").read({}, cache, [0, 1], [[1], [bad]])
    refused("answers for 3 prompts", cache, [[1], [2]], [[[3]], [[4]], [[5]]], None)
    rollout.Decoder(SHAPE, device="cpu")._check_score(cache, [[0, 300], [2]], [[[300]]])


def test_a_step_reads_no_length_past_the_cache(monkeypatch):
    """A slot past the cache is skipped and reported by the cache's calls; torch's indexing would end the
    GPU's context.  (Here with the cache's calls left out, on the CPU, where such an index raises.)"""
    for name in ("cache_grow", "cache_append"):
        monkeypatch.setattr(copes, name, lambda *a, **kw: None)
    monkeypatch.setattr(copes, "paged_attention", lambda cache, l, q, **kw: (torch.zeros_like(q), None))
    d = rollout.Decoder(SHAPE, device="cpu")
    w = torch.zeros(d.offsets[-1] + d.tensors[-1].numel)
    slots = torch.tensor([0, 4, -1, 2**31 - 1, -2**31], dtype=torch.int32)
    logits = d.step(d.weights(w), cache_of(8, 4, 4, 2), slots, torch.zeros(5, dtype=torch.int64))
    assert logits.shape == (5, 301) and slots.tolist() == [0, 4, -1, 2**31 - 1, -2**31]


def test_pages_that_a_score_needs_are_those_it_takes():
    """Against the pages in use when every answer is written, by the model of the bookkeeping."""
    rng = random.Random(7)
    for _ in range(200):
        size = rng.choice([1, 3, 7, 16])
        prompts = [[1] * rng.randint(1, 40) for _ in range(rng.randint(1, 4))]
        answers = [[[2] * rng.randint(1, 20) for _ in range(rng.randint(0, 3))] for _ in prompts]
        answers[0].append([2])
        n = len(prompts) + sum(map(len, answers))
        m = model.CacheModel(4000, size, n, 100)
        assert m.grow(range(len(prompts)), [len(p) for p in prompts]) == 0
        parents = [i for i, group in enumerate(answers) for _ in group]
        children = list(range(len(prompts), n))
        assert m.fork(parents, children) == 0
        assert m.grow(children, [len(a) - 1 for group in answers for a in group]) == 0
        need, longest = sum(r != 0 for r in m.refs), max(m.length)
        d = rollout.Decoder(SHAPE, device="cpu")
        d._check_score(cache_of(need, size, n, -(-longest // size)), prompts, answers)
        for few in (cache_of(need - 1, size, n, 100), cache_of(need, size, n - 1, 100),
                    cache_of(need, 1, n, longest - 1)):
            if few.desc.n_pages and few.desc.n_slots and few.desc.table_width:
                with pytest.raises(ValueError):
                    d._check_score(few, prompts, answers)
