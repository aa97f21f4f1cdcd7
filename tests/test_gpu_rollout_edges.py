"""Drawn rollouts at the edges: every token of every cut against the whole-number model, and what a decoder leaves in a
cache where it refuses or fails."""
import numpy as np
import pytest
import torch

import step_model as model
from test_gpu_rollout_sample import SHAPES, setup, uniform

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [dict(min_p=1.0), dict(min_p=1.0, top_k=5), dict(min_p=0.3), dict(min_p=0.05, top_p=0.9),
                                dict(min_p=0.2, temperature=1.7), dict(min_p=0.01, top_k=40, top_p=0.99, temperature=0.6), dict()])
def test_rollouts_token_by_token(kw):
    """The logits of the same steps give the tokens that were drawn, and their log probabilities within 2^-21 of themselves: two
    terms of one sign, each off by less than 2^-22.  min_p 1 keeps the largest logit's equals alone."""
    copes, decoder, layout, arena, prompts = setup(torch.bfloat16, **SHAPES[0])
    cache = decoder.cache(n_slots=4, max_tokens=40)
    n_tokens, u = 8, uniform(8, 4, seed=11)
    tokens, logprob = decoder.sample(arena.live, cache, prompts, n_tokens, u, **kw)
    assert not cache.length.any() and not cache.refs.any()
    args = {**dict(top_k=0, top_p=1.0, min_p=0.0, temperature=1.0), **kw}
    weights, slots = decoder.weights(arena.live), torch.arange(4, dtype=torch.int32, device="cuda")
    logits = decoder.read(weights, cache, range(4), prompts)
    for t in range(n_tokens):
        x = logits.float().cpu().numpy()
        for i in range(4):
            want, lp, kept = model.sample(x[i], float(u[t, i]), args["top_k"], args["top_p"], args["min_p"],
                                          float(np.float32(1.0 / args["temperature"])))
            got, got_lp = int(tokens[i, t]), float(logprob[i, t])
            assert got == want and abs(got_lp - lp) <= 2.0**-21 * abs(lp), (kw, t, i)
            if args["min_p"] == 1.0:
                ties = min(int((x[i] == x[i].max()).sum()), args["top_k"] or 301)
                assert x[i, got] == x[i].max() and kept == ties and abs(got_lp + np.log(ties)) <= 2.0**-20 * np.log(ties)
        logits = decoder.step(weights, cache, slots, tokens[:, t])
    copes.cache_free(cache, slots)
    copes.check()


def test_a_cache_that_is_refused_or_fails_is_empty():
    copes, decoder, layout, arena, prompts = setup(torch.float32, **SHAPES[0])
    u = uniform(3, 8)
    for dtype in (torch.float8_e4m3fn, torch.bfloat16):
        cache = decoder.cache(n_slots=12, max_tokens=40, dtype=dtype)
        for call in (lambda: decoder.sample(arena.live, cache, prompts, 3, u, rollouts=2), lambda: decoder.greedy(arena.live, cache, prompts, 3),
                     lambda: decoder.score(arena.live, cache, prompts, [[[1, 2]]])):
            with pytest.raises(ValueError):
                call()
            assert not cache.length.any() and not cache.refs.any()
    cache = decoder.cache(n_slots=12, max_tokens=40, dtype=torch.float32)
    want = decoder.sample(arena.live, cache, prompts, 3, u, rollouts=2)
    step, steps = decoder.step, []

    def failing(*args, **kw):
        steps.append(0)
        if len(steps) == 24:  # the prompts are read and forked
            raise RuntimeError("a step that fails")
        return step(*args, **kw)

    decoder.step = failing
    with pytest.raises(RuntimeError, match="a step that fails"):
        decoder.sample(arena.live, cache, prompts, 3, u, rollouts=2)
    assert len(steps) == 24 and not cache.length.any() and not cache.refs.any()
    got = decoder.sample(arena.live, cache, prompts, 3, u, rollouts=2)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    copes.check()
