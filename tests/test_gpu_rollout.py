"""A population judged by what it answers: rewards of a visit, and greedy continuations, against a
decoder in 64 bits that attends over whole sequences and shares nothing with the package's."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


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
        x = x + torch.einsum("hij,jhd->ihd", torch.softmax(z, -1), v).reshape(n, -1) @ get(f"l{l}.o", hidden, -1).T
        h = norm(x, get(f"l{l}.post_norm"))
        gate, up = h @ get(f"l{l}.gate", s.mlp, hidden).T, h @ get(f"l{l}.up", s.mlp, hidden).T
        x = x + (gate * torch.sigmoid(gate) * up) @ get(f"l{l}.down", hidden, s.mlp).T
    return norm(x, get("final_norm")) @ get("embed" if s.tied else "lm_head", s.vocab, hidden).T


def setup(dtype, **kw):
    from paper_2608_02391_gb300 import copes, rollout
    shape = rollout.Shape(2, 48, 80, 301, **kw)
    decoder = rollout.Decoder(shape)
    layout = copes.Layout([t.numel for t in decoder.tensors])
    rng = np.random.default_rng(5)
    theta = np.zeros(layout.d_pad, np.float32)
    for t, at in zip(decoder.tensors, decoder.offsets):
        theta[at:at + t.numel] = 1.0 + 0.1 * rng.standard_normal(t.numel) if t.kind == "norm" else \
            rng.standard_normal(t.numel) * (0.3 if t.kind == "embed" else 0.15)
    master = torch.from_numpy(theta).cuda()
    arena = copes.Arena(master.to(dtype, copy=True), master)
    prompts = [rng.integers(0, 301, k).tolist() for k in (5, 1, 16, 23)]
    answers = [[rng.integers(0, 301, k).tolist() for k in ks] for ks in ((3, 1, 9), (4,), (17, 2), (1, 1))]
    return copes, rollout, decoder, layout, arena, prompts, answers


def plain_score(shape, w, prompts, answers):
    out = []
    for p, group in zip(prompts, answers):
        for a in group:
            lp = torch.log_softmax(plain_logits(shape, w, p + a[:-1]), -1)
            out.append(float(np.mean([lp[len(p) - 1 + t, x].item() for t, x in enumerate(a)])))
    return np.array(out)


@pytest.mark.parametrize("kw", [dict(q_heads=6, kv_heads=2, head_dim=16, qkv_bias=True),
                                dict(q_heads=4, kv_heads=4, head_dim=8, qk_norm=True, tied=False)])
def test_rewards_of_a_visit_are_the_answers_log_probabilities(kw):
    """fp32 weights, so that the two decoders differ by rounding alone: a few hundred fp32 roundings
    (2^-24) of logits of a few units each, held to 2^-13 = 1.2e-4."""
    copes, rollout, decoder, layout, arena, prompts, answers = setup(torch.float32, **kw)
    from paper_2608_02391_gb300 import es
    cache = decoder.cache(n_slots=4 + 8, max_tokens=48, page_size=16, dtype=torch.float32)
    sub = copes.tiles_from_ranges([(0, layout.d_pad)], tile_size=4096)
    cfg = es.ESConfig(n_members=6, sigma=1e-2, alpha=5e-3)
    rewards, plain = torch.empty(6, device="cuda"), []

    def evaluate(i):
        got = decoder.score(arena.live, cache, prompts, answers)
        rewards[i] = got.mean()
        want = plain_score(decoder.shape, arena.live, prompts, answers)
        assert np.abs(got.double().cpu().numpy() - want).max() <= 2.0**-13
        plain.append(want.mean())
        assert not cache.refs.any() and not cache.length.any()

    before = arena.master.clone()
    es.round_robin_visit(arena, sub, 0, 0, cfg, layout.d_pad, rewards, evaluate=evaluate)
    copes.check()
    assert len(plain) == 6 and np.std(plain) > 1e-3
    assert np.allclose(rewards.double().cpu().numpy(), plain, rtol=0, atol=2.0**-13)
    assert not torch.equal(before, arena.master)


def test_greedy_continuations_and_bf16():
    """fp32: the tokens of the 64-bit decoder wherever its two best logits are further apart than the
    rounding.  bf16: the scores within 2^-4 of the 64-bit decoder's on the same weights."""
    copes, rollout, decoder, layout, arena, prompts, answers = setup(torch.float32, q_heads=6, kv_heads=2, head_dim=16)
    cache = decoder.cache(n_slots=12, max_tokens=48, dtype=torch.float32)
    got = decoder.greedy(arena.w, cache, prompts, 6).tolist()
    for p, tokens in zip(prompts, got):
        seq = list(p)
        for t in tokens:
            logits = plain_logits(decoder.shape, arena.w, seq)[-1]
            assert logits[t] >= logits.max() - 2.0**-13
            seq.append(t)
    copes.check()
    half = arena.w.bfloat16()
    cache = decoder.cache(n_slots=12, max_tokens=48)
    got = decoder.score(half, cache, prompts, answers).double().cpu().numpy()
    assert np.abs(got - plain_score(decoder.shape, half, prompts, answers)).max() <= 2.0**-4
    copes.check()


def test_scores_need_the_pages_they_take_and_no_more(monkeypatch):
    """Exactly enough pages give the scores that plenty of them give; one less is refused, before any work or,
    where that check is left out, by the report of the page that a kernel did not find."""
    copes, rollout, decoder, layout, arena, prompts, answers = setup(torch.float32, q_heads=6, kv_heads=2, head_dim=16)
    plenty = decoder.cache(n_slots=13, max_tokens=48, dtype=torch.float32)
    want = decoder.score(arena.w, plenty, prompts, answers)
    # pages of 16: prompts of 5, 1, 16, 23 take 1 + 1 + 1 + 2; answers 1 + 1 + 1; 1; 1 + 1; 1 + 1
    for spare in (0, 1):  # a page of another sequence
        cache = decoder.cache(n_slots=13, max_tokens=48, n_pages=13 + spare, dtype=torch.float32)
        last = torch.tensor([12], dtype=torch.int32, device="cuda")
        copes.cache_grow(cache, last, spare)
        assert torch.equal(decoder.score(arena.w, cache, prompts, answers), want)
        assert cache.refs.sum().item() == spare
        short = decoder.cache(n_slots=13, max_tokens=48, n_pages=12 + spare, dtype=torch.float32)
        copes.cache_grow(short, last, spare)
        with pytest.raises(ValueError, match="pages"):
            decoder.score(arena.w, short, prompts, answers)
        assert short.refs.sum().item() == spare
    monkeypatch.setattr(rollout.Decoder, "_check_room", lambda *a: None)
    with pytest.raises(copes.CopesError, match="bits 0x40:"):
        decoder.score(arena.w, short, prompts, answers)
    copes.check()
