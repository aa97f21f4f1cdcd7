"""Drawn rollouts of a decoder on the arena's weights: with norms around its blocks, against a decoder in 64 bits, with a cache in
8 bits, and as the rewards of a visit."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

SHAPES = [dict(q_heads=6, kv_heads=2, head_dim=16, qkv_bias=True),
          dict(q_heads=4, kv_heads=4, head_dim=16, qk_norm=True, tied=False, out_norms=True, block_gates=True, residual_scale=0.7),
          dict(q_heads=6, kv_heads=2, head_dim=16, out_norms=True)]


def plain_logits(shape, w, tokens):
    """Logits [tokens, vocab] in float64 of one sequence, by the definition."""
    s, w = shape, w.detach().double().cpu()
    offsets, at = {}, 0
    for t in s.tensors():
        offsets[t.name] = (at, t.numel)
        at = (at + t.numel + 63) // 64 * 64
    get = lambda name, *dims: w[offsets[name][0]:offsets[name][0] + offsets[name][1]].view(*dims or (-1,))
    norm = lambda x, g: x / torch.sqrt((x * x).mean(-1, keepdim=True) + s.eps) * g
    n, d, hidden = len(tokens), s.head_dim, s.hidden
    angle = torch.arange(n, dtype=torch.float64)[:, None] * s.rope_base ** -(torch.arange(0, d, 2, dtype=torch.float64) / d)

    def rotate(x):  # [n, heads, d]
        c, sn = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        a, b = x[..., :d // 2], x[..., d // 2:]
        return torch.cat((a * c - b * sn, b * c + a * sn), -1)

    def after(x, y, block):
        if s.out_norms:
            y = norm(y, get(block + "_out_norm"))
        if s.block_gates:
            y = y * get(block + "_gate")
        return x + s.residual_scale * y

    x = get("embed", s.vocab, hidden)[torch.tensor(tokens)]
    for l in range(s.layers):
        h = norm(x, get(f"l{l}.in_norm"))
        q, k, v = (h @ get(f"l{l}.{m}", -1, hidden).T + (get(f"l{l}.{m}_bias") if s.qkv_bias else 0) for m in "qkv")
        q, k, v = (y.view(n, -1, d) for y in (q, k, v))
        if s.qk_norm:
            q, k = norm(q, get(f"l{l}.q_norm")), norm(k, get(f"l{l}.k_norm"))
        q, k = rotate(q), rotate(k)
        k, v = (y.repeat_interleave(s.q_heads // s.kv_heads, 1) for y in (k, v))
        z = torch.einsum("ihd,jhd->hij", q, k) * d ** -0.5
        z = z.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -torch.inf)
        x = after(x, torch.einsum("hij,jhd->ihd", torch.softmax(z, -1), v).reshape(n, -1) @ get(f"l{l}.o", hidden, -1).T, f"l{l}.attn")
        h = norm(x, get(f"l{l}.post_norm"))
        gate, up = h @ get(f"l{l}.gate", s.mlp, hidden).T, h @ get(f"l{l}.up", s.mlp, hidden).T
        x = after(x, (gate * torch.sigmoid(gate) * up) @ get(f"l{l}.down", hidden, s.mlp).T, f"l{l}.mlp")
    return norm(x, get("final_norm")) @ get("embed" if s.tied else "lm_head", s.vocab, hidden).T


def setup(dtype, fused=False, **kw):
    from paper_2608_02391_gb300 import copes, rollout
    decoder = rollout.Decoder(rollout.Shape(2, 48, 80, 301, **kw), fused=fused)
    layout = copes.Layout([t.numel for t in decoder.tensors])
    rng = np.random.default_rng(5)
    theta = np.zeros(layout.d_pad, np.float32)
    for t, at in zip(decoder.tensors, decoder.offsets):
        theta[at:at + t.numel] = 1.0 + 0.1 * rng.standard_normal(t.numel) if t.kind == "norm" else \
            rng.standard_normal(t.numel) * (0.3 if t.kind == "embed" else 0.15)
    master = torch.from_numpy(theta).cuda()
    arena = copes.Arena(master.to(dtype, copy=True), master)
    prompts = [rng.integers(0, 301, k).tolist() for k in (5, 1, 16, 23)]
    return copes, decoder, layout, arena, prompts


def uniform(n_tokens, n, seed=0):
    return torch.rand(n_tokens, n, device="cuda", generator=torch.Generator("cuda").manual_seed(seed))


@pytest.mark.parametrize("kw", SHAPES)
def test_drawn_rollouts_follow_the_decoder_in_64_bits(kw):
    """fp32 weights: log probabilities of drawn tokens within 2^-13, as a few hundred fp32 roundings (2^-24) of logits of a few units
    each leave them; and each token is the one that its number points at, where it is further than that from the borders."""
    copes, decoder, layout, arena, prompts = setup(torch.float32, fused=True, **kw)
    cache = decoder.cache(n_slots=4 + 12, max_tokens=40, page_size=4, dtype=torch.float32)
    u = uniform(7, 12)
    tokens, logprob = decoder.sample(arena.live, cache, prompts, 7, u, rollouts=3, temperature=0.8)
    assert not cache.refs.any() and not cache.length.any()
    seen = 0
    for i in range(12):
        p, row = prompts[i // 3], tokens[i].tolist()
        z = plain_logits(decoder.shape, arena.live, p + row[:-1])[len(p) - 1:] / 0.8
        lp = torch.log_softmax(z, -1)
        want = lp[torch.arange(7), torch.tensor(row)]
        assert (logprob[i].double().cpu() - want).abs().max() <= 2.0**-13
        sums = torch.cumsum(torch.exp(lp), -1)
        for t, x in enumerate(row):
            at, low, high = float(u[t, i]), float(sums[t, x - 1]) if x else 0.0, float(sums[t, x])
            assert low - 2.0**-13 <= at < high + 2.0**-13
            seen += low + 2.0**-13 < at < high - 2.0**-13
    assert seen > 60  # of 84: the others are near a border
    score = decoder.score(arena.live, cache, prompts, [[r.tolist() for r in tokens[3 * i:3 * i + 3]] for i in range(4)])
    assert torch.isfinite(score).all()


@pytest.mark.parametrize("kw", SHAPES)
def test_scores_with_fused_norms(kw):
    copes, decoder, layout, arena, prompts = setup(torch.float32, fused=True, **kw)
    rng = np.random.default_rng(6)
    answers = [[rng.integers(0, 301, k).tolist() for k in ks] for ks in ((3, 1, 9), (4,), (17, 2), (1, 1))]
    cache = decoder.cache(n_slots=12, max_tokens=48, page_size=16, dtype=torch.float32)
    got = decoder.score(arena.live, cache, prompts, answers).double().cpu().numpy()
    want = []
    for p, group in zip(prompts, answers):
        for a in group:
            lp = torch.log_softmax(plain_logits(decoder.shape, arena.live, p + a[:-1]), -1)
            want.append(float(np.mean([lp[len(p) - 1 + t, x].item() for t, x in enumerate(a)])))
    assert np.abs(got - want).max() <= 2.0**-13


def test_the_likeliest_token_alone_is_the_greedy_continuation():
    copes, decoder, layout, arena, prompts = setup(torch.bfloat16, **SHAPES[0])
    cache = decoder.cache(n_slots=4, max_tokens=40)
    greedy = decoder.greedy(arena.live, cache, prompts, 6)
    for kw in (dict(top_k=1), dict(top_p=1e-6), dict(min_p=1.0, top_k=5)):
        tokens, logprob = decoder.sample(arena.live, cache, prompts, 6, uniform(6, 4), **kw)
        if kw.get("min_p"):
            continue  # equal logits are all kept
        assert torch.equal(tokens, greedy) and not logprob.any()


def test_the_same_numbers_give_the_same_rollouts():
    copes, decoder, layout, arena, prompts = setup(torch.bfloat16, fused=True, **SHAPES[1])
    cache = decoder.cache(n_slots=4 + 20, max_tokens=40, page_size=8)
    u = uniform(9, 20, seed=3)
    first = decoder.sample(arena.live, cache, prompts, 9, u, rollouts=5, top_p=0.95)
    again = decoder.sample(arena.live, cache, prompts, 9, u, rollouts=5, top_p=0.95)
    other = decoder.sample(arena.live, cache, prompts, 9, uniform(9, 20, seed=4), rollouts=5, top_p=0.95)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1]) and not torch.equal(first[0], other[0])
    with pytest.raises(copes.CopesError):
        bad = u.clone()
        bad[4, 3] = 1.0
        decoder.sample(arena.live, cache, prompts, 9, bad, rollouts=5)
    assert not cache.refs.any() and not cache.length.any()


@pytest.mark.parametrize("kw", SHAPES[:2])
def test_rollouts_with_a_cache_in_8_bits(kw):
    copes, decoder, layout, arena, prompts = setup(torch.bfloat16, fused=True, **kw)
    cache = decoder.cache(n_slots=4 + 8, max_tokens=40, page_size=8, dtype=torch.float8_e4m3fn)
    tokens, logprob = decoder.sample(arena.live, cache, prompts, 6, uniform(6, 8), rollouts=2, top_k=40)
    assert torch.isfinite(logprob).all() and (logprob <= 0).all() and ((tokens >= 0) & (tokens < 301)).all()
    answers = [[tokens[2 * i].tolist(), tokens[2 * i + 1].tolist()] for i in range(4)]
    scores = decoder.score(arena.live, cache, prompts, answers)
    assert torch.isfinite(scores).all() and decoder.greedy(arena.live, cache, prompts, 3).shape == (4, 3)
    assert not cache.refs.any() and not cache.length.any()
    # what a step writes is what the same step writes in 16 bits, rounded
    import step_model
    whole = decoder.cache(n_slots=4, max_tokens=40, page_size=8)
    weights, rows, first = decoder.weights(arena.live), torch.arange(4, dtype=torch.int32, device="cuda"), torch.tensor([1, 2, 3, 4], device="cuda")
    decoder.step(weights, cache, rows, first)
    decoder.step(weights, whole, rows, first)
    for got, want in zip(copes.cache_read(cache, 0, slots=rows), copes.cache_read(whole, 0, slots=rows)):
        assert np.array_equal(got.double().cpu().numpy(), step_model.stored(want.double().cpu().numpy())[0])
    copes.check()


def test_a_visit_rewarded_by_drawn_answers():
    copes, decoder, layout, arena, prompts = setup(torch.bfloat16, fused=True, **SHAPES[2])
    from paper_2608_02391_gb300 import es
    cache = decoder.cache(n_slots=4 + 16, max_tokens=32, page_size=8, dtype=torch.float8_e4m3fn)
    sub = copes.tiles_from_ranges([(0, layout.d_pad)], tile_size=4096)
    cfg = es.ESConfig(n_members=4, sigma=1e-2, alpha=5e-3)
    rewards, u = torch.empty(4, device="cuda"), uniform(5, 16)

    def evaluate(i):  # how often an even token was drawn
        tokens, _ = decoder.sample(arena.live, cache, prompts, 5, u, rollouts=4, temperature=1.2, top_p=0.99)
        rewards[i] = (tokens % 2 == 0).float().mean()

    before = arena.master.clone()
    es.round_robin_visit(arena, sub, 0, 0, cfg, layout.d_pad, rewards, evaluate=evaluate)
    copes.check()
    assert ((rewards >= 0) & (rewards <= 1)).all() and not torch.equal(arena.master, before)


@pytest.mark.parametrize("fused", [False, True])
def test_a_decoder_without_layers(fused):
    from paper_2608_02391_gb300 import copes, rollout
    decoder = rollout.Decoder(rollout.Shape(0, 48, 80, 301, 4, 2, 16), fused=fused)
    cache = copes.KVCache.empty(4, 1, 2, 16, 16, 2, 2, dtype=torch.float32)
    w = torch.randn(decoder.offsets[-1] + 48, device="cuda")
    weights = decoder.weights(w)
    slots, tokens = torch.arange(2, dtype=torch.int32, device="cuda"), torch.tensor([7, 300], device="cuda")
    logits = decoder.step(weights, cache, slots, tokens)
    x = w[:301 * 48].view(301, 48).double()
    h = x[tokens] / torch.sqrt((x[tokens] ** 2).mean(-1, keepdim=True) + 1e-6) * weights["final_norm"].double()
    # a product off by 10 half steps of 2^-24 at most, its norm among them, and 48 roundings of their sum
    assert ((logits - h @ x.T).abs() <= 60 * 2.0**-24 * (h.abs() @ x.abs().T)).all()
    assert decoder.step(weights, cache, slots, tokens, logits=False) is None
    copes.check()
