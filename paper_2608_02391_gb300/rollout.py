"""Rewards of a population from what its members answer: a decoder that reads its weights from the
arena under evolution.

The layouts of ``workloads.decoder_tensors`` are decoders: token embedding, layers of grouped-query
attention with rotary positions and a gated MLP, and a head.  ``Decoder`` runs one for single tokens
on a flat weight buffer -- ``arena.live`` while a member is evaluated -- with torch's matrix products
and the library's cache, attention and log probabilities:

score   mean log probability of given answers, the answers of one prompt sharing the prompt's pages
        (cache_fork): a dense reward that needs no sampling
greedy  the likeliest continuation of each prompt, for a verifier to judge

One visit with answers as rewards:

    decoder = rollout.Decoder(rollout.Shape(24, 896, 4864, 151936, 14, 2, 64, qkv_bias=True))
    cache = decoder.cache(n_slots=64, max_tokens=512)

    def evaluate(i):                                   # runs while member i is live
        rewards[i] = decoder.score(arena.live, cache, prompts, answers).mean()

    es.round_robin_visit(arena, subs[k], k, iteration, cfg, layout.d_pad, rewards, evaluate=evaluate)
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Dict, List, Sequence

import torch

from . import copes, workloads


@dataclass(frozen=True)
class Shape:
    """The arguments of workloads.decoder_tensors, and the base of the rotary frequencies."""
    layers: int
    hidden: int
    mlp: int
    vocab: int
    q_heads: int
    kv_heads: int
    head_dim: int
    qkv_bias: bool = False
    qk_norm: bool = False
    tied: bool = True
    rope_base: float = 1e6
    eps: float = 1e-6

    def tensors(self) -> List[workloads.Tensor]:
        return workloads.decoder_tensors(self.layers, self.hidden, self.mlp, self.vocab, self.q_heads, self.kv_heads,
                                         self.head_dim, self.qkv_bias, self.qk_norm, self.tied)


def _rms_norm(x: torch.Tensor, weight: torch.Tensor, eps: float) -> torch.Tensor:
    f = x.float()
    return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + eps)).to(x.dtype) * weight


class Decoder:
    """A decoder over flat weight buffers with the layout of shape.tensors()."""

    def __init__(self, shape: Shape, device="cuda"):
        self.shape = shape
        self.tensors = shape.tensors()
        self.offsets = workloads.layout_offsets(self.tensors)
        half = torch.arange(0, shape.head_dim, 2, device=device, dtype=torch.float64) / shape.head_dim
        self.frequencies = shape.rope_base ** -half

    def weights(self, w: torch.Tensor) -> Dict[str, torch.Tensor]:
        """Views of the flat buffer: matrices as [out, in], vectors flat."""
        s = self.shape
        q, kv = s.q_heads * s.head_dim, s.kv_heads * s.head_dim
        out_in = {"embed": (s.vocab, s.hidden), "lm_head": (s.vocab, s.hidden), "q": (q, s.hidden), "k": (kv, s.hidden),
                  "v": (kv, s.hidden), "o": (s.hidden, q), "gate": (s.mlp, s.hidden), "up": (s.mlp, s.hidden),
                  "down": (s.hidden, s.mlp)}
        views = {}
        for t, at in zip(self.tensors, self.offsets):
            flat = w[at:at + t.numel]
            shape = out_in.get(t.name.rsplit(".", 1)[-1])
            views[t.name] = flat if shape is None else flat.view(shape)
        return views

    def cache(self, n_slots: int, max_tokens: int, page_size: int = 16, n_pages: int = 0, dtype=torch.bfloat16,
              device="cuda") -> copes.KVCache:
        """An empty cache of n_slots sequences of up to max_tokens (n_pages: fewer pages than all of
        them need, where many share a prompt)."""
        s, width = self.shape, -(-max_tokens // page_size)
        return copes.KVCache.empty(n_pages or n_slots * width, s.layers, s.kv_heads, page_size, s.head_dim, n_slots, width,
                                   dtype=dtype, device=device)

    def _rotate(self, x: torch.Tensor, angles: torch.Tensor) -> torch.Tensor:
        """Rotary positions of x [n, heads, head_dim] by angles [n, head_dim / 2]: the halves of a head are the pairs."""
        cos, sin = (f(angles).float()[:, None] for f in (torch.cos, torch.sin))
        a, b = x.float().chunk(2, -1)
        return torch.cat((a * cos - b * sin, b * cos + a * sin), -1).to(x.dtype)

    def step(self, weights: Dict[str, torch.Tensor], cache: copes.KVCache, slots: torch.Tensor, tokens: torch.Tensor,
             logits: bool = True):
        """The next token of each of `slots` (distinct, int32) is tokens (int64, in the vocabulary): their logits [n, vocab],
        or None where they are not asked for.  Slots past the cache, and tokens that it has no room for, are
        reported by copes.check()."""
        s, n = self.shape, slots.numel()
        copes.cache_grow(cache, slots, 1)
        place = cache.length[slots.long().clamp_(0, cache.desc.n_slots - 1)] - 1  # a slot past the cache is the calls' to report
        angles = place.double()[:, None] * self.frequencies
        x = weights["embed"][tokens]
        for l in range(s.layers):
            get = lambda name: weights.get(f"l{l}.{name}")
            h = _rms_norm(x, get("in_norm"), s.eps)
            q, k, v = (torch.nn.functional.linear(h, get(m), get(m + "_bias")).view(n, -1, s.head_dim) for m in "qkv")
            if s.qk_norm:
                q, k = _rms_norm(q, get("q_norm"), s.eps), _rms_norm(k, get("k_norm"), s.eps)
            copes.cache_append(cache, l, self._rotate(k, angles), v, slots=slots)
            out, _ = copes.paged_attention(cache, l, self._rotate(q, angles), slots=slots)
            x = x + out.flatten(1) @ get("o").T
            h = _rms_norm(x, get("post_norm"), s.eps)
            x = x + (torch.nn.functional.silu(h @ get("gate").T) * (h @ get("up").T)) @ get("down").T
        if not logits:
            return None
        return _rms_norm(x, weights["final_norm"], s.eps) @ weights["embed" if s.tied else "lm_head"].T

    def _check_tokens(self, what: str, sequences: Sequence[Sequence[int]]) -> None:
        """Raises for no sequences, for one without tokens, whose reward would be 0 / 0, and for an id outside the
        vocabulary: a negative one would be read as another token, one past it end the GPU's context."""
        if len(sequences) == 0:
            raise ValueError(f"no {what}s")
        if min(map(len, sequences)) == 0:
            raise ValueError(f"an empty {what}")
        if min(map(min, sequences)) < 0 or max(map(max, sequences)) >= self.shape.vocab:
            raise ValueError(f"a token outside the vocabulary of {self.shape.vocab} in the {what}s")

    def read(self, weights: Dict[str, torch.Tensor], cache: copes.KVCache, slots: Sequence[int],
             prompts: Sequence[Sequence[int]]) -> torch.Tensor:
        """Writes prompts (one token at least each) into empty slots and returns the logits after each."""
        self._check_tokens("prompt", prompts)
        device = cache.pool.device
        last = [None] * len(prompts)
        for t in range(max(map(len, prompts))):
            rows = [i for i, p in enumerate(prompts) if t < len(p)]
            ends = [i for i in rows if t + 1 == len(prompts[i])]
            logits = self.step(weights, cache, torch.tensor([slots[i] for i in rows], dtype=torch.int32, device=device),
                               torch.tensor([prompts[i][t] for i in rows], device=device), logits=bool(ends))
            for i in ends:
                last[i] = logits[rows.index(i)]
        return torch.stack(last)

    def _check_room(self, cache: copes.KVCache, lengths: Sequence[int], pages: int) -> None:
        """Raises where sequences of these lengths, in `pages` pages that are not there yet, have no room in the
        first slots of the cache.  The cache's calls refuse on the device, and what is computed after that
        would be a reward like any other."""
        d = cache.desc
        if len(lengths) > d.n_slots:
            raise ValueError(f"{len(lengths)} sequences in a cache of {d.n_slots} slots")
        if max(lengths) > d.table_width * d.page_size:
            raise ValueError(f"a sequence of {max(lengths)} tokens in a cache of up to {d.table_width * d.page_size}")
        begun, used = torch.stack((cache.length[:len(lengths)].count_nonzero(), cache.refs.count_nonzero())).tolist()
        if begun:
            raise ValueError(f"{begun} of the cache's first {len(lengths)} slots are not empty")
        if used + pages > d.n_pages:
            raise ValueError(f"{pages} pages are needed, and {d.n_pages - used} of the cache's {d.n_pages} are free")

    def _check_score(self, cache: copes.KVCache, prompts: Sequence[Sequence[int]],
                     answers: Sequence[Sequence[Sequence[int]]]) -> None:
        self._check_tokens("prompt", prompts)
        if len(answers) > len(prompts):
            raise ValueError(f"answers for {len(answers)} prompts, and {len(prompts)} prompts")
        self._check_tokens("answer", [a for group in answers for a in group])
        size, prompt = cache.desc.page_size, [len(p) for p in prompts]
        pages = sum(-(-p // size) for p in prompt)
        lengths = list(prompt)
        for p, group in zip(prompt, answers):
            for a in group:  # its last token is not written; the prompt's full pages are shared
                lengths.append(p + len(a) - 1)
                pages += -(-lengths[-1] // size) - p // size
        self._check_room(cache, lengths, pages)

    def score(self, w: torch.Tensor, cache: copes.KVCache, prompts: Sequence[Sequence[int]],
              answers: Sequence[Sequence[Sequence[int]]]) -> torch.Tensor:
        """Mean log probability of every answer under the weights w: fp32, the answers of prompt 0,
        then those of prompt 1, ...  The cache's first slots, one for each prompt and each answer, are
        empty before and after.  Prompts or answers without tokens, ids outside the vocabulary, answers without
        a prompt and what the cache has no room for raise ValueError before any work; what a kernel reports
        (copes.check), CopesError."""
        self._check_score(cache, prompts, answers)
        weights, device = self.weights(w), cache.pool.device
        flat = [(i, a) for i, group in enumerate(answers) for a in group]
        n, first = len(flat), len(prompts)
        slots = list(range(first))
        logits = self.read(weights, cache, slots, prompts)
        parents = torch.tensor([i for i, _ in flat], dtype=torch.int32, device=device)
        children = torch.arange(first, first + n, dtype=torch.int32, device=device)
        copes.cache_fork(cache, parents, children)
        width = max(len(a) for _, a in flat)
        table = torch.full((width, n), -1, dtype=torch.int64)
        for j, (_, a) in enumerate(flat):
            table[:len(a), j] = torch.tensor(a)
        table = table.to(device)
        total = copes.token_logprobs(logits[parents.long()], table[0]).logprob
        lengths = torch.tensor([len(a) for _, a in flat])
        for t in range(1, width):  # after token t - 1, for the answers that have a token t
            rows = (lengths > t).nonzero()[:, 0].to(device)
            logits = self.step(weights, cache, children[rows], table[t - 1, rows])
            total[rows] += copes.token_logprobs(logits, table[t, rows]).logprob
        copes.cache_free(cache, torch.arange(first + n, dtype=torch.int32, device=device))
        copes.check()
        return total / lengths.to(device)

    def greedy(self, w: torch.Tensor, cache: copes.KVCache, prompts: Sequence[Sequence[int]], n_tokens: int) -> torch.Tensor:
        """The n_tokens likeliest next tokens of each prompt, one after the other: int64 [prompts,
        n_tokens].  The cache's first slots, one for each prompt, are empty before and after; errors as score's."""
        self._check_tokens("prompt", prompts)
        if n_tokens < 1:
            raise ValueError(f"a continuation of {n_tokens} tokens")
        lengths = [len(p) + n_tokens - 1 for p in prompts]  # the last token is not written
        self._check_room(cache, lengths, sum(-(-k // cache.desc.page_size) for k in lengths))
        weights, device = self.weights(w), cache.pool.device
        slots = torch.arange(len(prompts), dtype=torch.int32, device=device)
        none = torch.full((len(prompts),), -1, dtype=torch.int64, device=device)
        logits, out = self.read(weights, cache, list(range(len(prompts))), prompts), []
        for t in range(n_tokens):
            out.append(copes.token_logprobs(logits, none, top=1).top_ids[:, 0])
            if t + 1 < n_tokens:
                logits = self.step(weights, cache, slots, out[-1])
        copes.cache_free(cache, slots)
        copes.check()
        return torch.stack(out, 1)
