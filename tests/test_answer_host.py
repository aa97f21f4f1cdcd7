"""Refusals of the answering operators' C entries: every case fails its checks before any CUDA
call, with a message that names the entry; the fake addresses are never read."""
import copy
import ctypes
import gc
import os
import weakref
from types import SimpleNamespace

import pytest
import torch

import answer_model as model

GOOD = dict(pool=0x1000000, dtype=0, n_pages=8, n_layers=2, n_kv_heads=2, page_size=16, head_dim=64, table=0x9000000,
            n_slots=4, table_width=5, length=0xA000000, refs=0xB000000)
WS, BIG = 0xC000000, 1 << 30


@pytest.fixture(scope="module")
def copes():
    from paper_2608_02391_gb300 import build, copes as c
    if not os.path.exists(c.LIB_PATH):
        build.build()
    c.load()
    return c


def cache(copes, **kw):
    f = copy.copy(GOOD)
    f.update(kw)
    return ctypes.byref(copes.KVCacheDesc(*[f[name] for name, _ in copes.KVCacheDesc._fields_]))


def calls(copes, c):
    """Every entry that takes a cache, with arguments that are fine where the cache is."""
    L = copes.load()
    return {
        "copes_cache_grow": lambda: L.copes_cache_grow(c, 0x100, 1, None, 1, WS, BIG, None),
        "copes_cache_append": lambda: L.copes_cache_append(c, 0, 0x100, None, 1, 0x100, 64, 64, 0x100, 64, 64, None),
        "copes_cache_fork": lambda: L.copes_cache_fork(c, 0x100, 0x200, 1, WS, BIG, None),
        "copes_cache_free": lambda: L.copes_cache_free(c, 0x100, 1, None),
        "copes_cache_compact": lambda: L.copes_cache_compact(c, None, WS, BIG, None),
        "copes_cache_copy_pages": lambda: L.copes_cache_copy_pages(c, 0x100, 0x200, 1, None),
        "copes_paged_attention": lambda: L.copes_paged_attention(c, 0, None, 1, 0x100, 256, 64, 4, 0.1, 0xD000000, None,
                                                                 WS, BIG, None),
    }


def refused(copes, rc, code, name):
    assert rc == code, (name, rc, copes.last_error())
    assert name in copes.last_error()


@pytest.mark.parametrize("change,code", [
    (dict(pool=None), -1), (dict(table=None), -1), (dict(length=None), -1), (dict(refs=None), -1), (dict(dtype=2), -1),
    (dict(n_pages=0), -1), (dict(n_layers=0), -1), (dict(n_kv_heads=-1), -1), (dict(page_size=0), -1), (dict(n_slots=0), -1),
    (dict(table_width=0), -1), (dict(head_dim=60), -3), (dict(head_dim=264), -3), (dict(head_dim=0), -3),
    (dict(n_pages=(1 << 22) + 1), -3), (dict(table_width=1 << 28), -3), (dict(n_slots=1 << 30, table_width=2), -3),
    (dict(n_layers=1 << 20), -3), (dict(page_size=1 << 24, head_dim=256, table_width=1, n_pages=1), -3),
    (dict(page_size=1 << 22, n_kv_heads=60000, n_layers=60000, table_width=1), -3),
    (dict(pool=0x1000008), -2), (dict(table=0x9000002), -2), (dict(length=0xA000001), -2), (dict(refs=0xB000003), -2),
    (dict(length=0x9000010), -1), (dict(refs=0x1000100), -1)])
def test_caches_that_are_refused(copes, change, code):
    c = cache(copes, **change)
    for name, call in calls(copes, c).items():
        refused(copes, call(), code, name)
    assert copes.load().copes_cache_workspace_bytes(c) == 0
    assert copes.load().copes_paged_attention_workspace_bytes(c, 1, 4) == 0


def test_a_null_cache_is_refused(copes):
    for name, call in calls(copes, None).items():
        refused(copes, call(), -1, name)


def test_arguments_that_are_refused(copes):
    L, c = copes.load(), cache(copes)
    ws = L.copes_cache_workspace_bytes(c)
    assert ws >= 4 * (2 * 8 + 2 * 4)

    def grow(slots=0x100, n=1, add=None, add_all=1, work=WS, size=BIG):
        return L.copes_cache_grow(c, slots, n, add, add_all, work, size, None)

    for kw, code in [(dict(slots=None), -1), (dict(n=-1), -1), (dict(n=5), -3), (dict(slots=0x102), -2), (dict(add=0x101), -2),
                     (dict(add_all=-1), -1), (dict(work=None), -4), (dict(size=ws - 1), -4), (dict(work=WS + 4), -2)]:
        refused(copes, grow(**kw), code, "copes_cache_grow")
    for kw, code in [((None, 0x200, 1), -1), ((0x100, None, 1), -1), ((0x100, 0x200, 5), -3), ((0x100, 0x201, 1), -2)]:
        refused(copes, L.copes_cache_fork(c, *kw, WS, BIG, None), code, "copes_cache_fork")
    refused(copes, L.copes_cache_fork(c, 0x100, 0x200, 1, WS, ws - 1, None), -4, "copes_cache_fork")
    refused(copes, L.copes_cache_free(c, None, 1, None), -1, "copes_cache_free")
    refused(copes, L.copes_cache_free(c, 0x100, -2, None), -1, "copes_cache_free")
    refused(copes, L.copes_cache_compact(c, 0x101, WS, BIG, None), -2, "copes_cache_compact")
    refused(copes, L.copes_cache_compact(c, None, WS, 16, None), -4, "copes_cache_compact")
    refused(copes, L.copes_cache_copy_pages(c, 0x100, None, 1, None), -1, "copes_cache_copy_pages")

    def append(layer=0, slots=0x100, position=None, n=1, k=0x100, v=0x100):
        return L.copes_cache_append(c, layer, slots, position, n, k, 64, 64, v, 64, 64, None)

    for kw, code in [(dict(layer=2), -1), (dict(layer=-1), -1), (dict(slots=None, n=5), -3), (dict(position=0x102), -2),
                     (dict(k=None), -1), (dict(v=None), -1), (dict(k=0x101), -2), (dict(n=-1), -1), (dict(k=0x1000010), -1),
                     (dict(v=0x1000010), -1)]:
        refused(copes, append(**kw), code, "copes_cache_append")

    need = L.copes_paged_attention_workspace_bytes(c, 4, 8)
    assert need > 0 and L.copes_paged_attention_workspace_bytes(c, 4, 7) == 0
    assert L.copes_paged_attention_workspace_bytes(c, -1, 8) == 0

    def attend(layer=0, slots=None, n=4, q=0x100, heads=8, scale=0.1, out=0xD000000, lse=None, work=WS, size=BIG):
        return L.copes_paged_attention(c, layer, slots, n, q, 512, 64, heads, scale, out, lse, work, size, None)

    for kw, code in [(dict(layer=2), -1), (dict(n=5), -3), (dict(n=-1), -1), (dict(q=None), -1), (dict(out=None), -1),
                     (dict(heads=7), -1), (dict(heads=0), -1), (dict(heads=70000), -3), (dict(scale=float("nan")), -1),
                     (dict(scale=float("inf")), -1), (dict(q=0x101), -2), (dict(out=0xD000008), -2), (dict(lse=0xE000002), -2),
                     (dict(out=0x1000010), -1), (dict(lse=0x1000010), -1), (dict(lse=0xD000010), -1), (dict(slots=0x102), -2),
                     (dict(q=0xD000004), -1), (dict(lse=0x200), -1),
                     (dict(work=None), -4), (dict(size=need - 1), -4), (dict(work=WS + 8), -2)]:
        refused(copes, attend(**kw), code, "copes_paged_attention")

    def logprobs(logits=0x100000, dtype=0, n=1, vocab=100, target=0x1000, scale=1.0, top=2, lp=0x2000, ent=None, ids=0x3000,
                 tlp=0x4000):
        return L.copes_token_logprobs(logits, dtype, n, vocab, 100, target, scale, top, lp, ent, ids, tlp, None)

    for kw, code in [(dict(dtype=2), -1), (dict(n=-1), -1), (dict(vocab=0), -1), (dict(vocab=(1 << 30) + 1), -3), (dict(scale=0.0), -1),
                     (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(top=-1), -3),
                     (dict(top=33), -3), (dict(vocab=1), -3), (dict(logits=None), -1), (dict(target=None), -1), (dict(lp=None), -1),
                     (dict(lp=0x100004), -1), (dict(ent=0x100004), -1), (dict(ids=0x100008), -1), (dict(tlp=0x1000C4), -1), (dict(ids=None), -1), (dict(tlp=None), -1), (dict(logits=0x101), -2), (dict(target=0x1004), -2),
                     (dict(ids=0x3004), -2), (dict(lp=0x2002), -2), (dict(ent=0x5001), -2)]:
        refused(copes, logprobs(**kw), code, "copes_token_logprobs")


def test_arguments_in_the_cache_or_in_one_another_are_refused(copes):
    """Each in the last byte of what it must not share, and read-only lists where they may lie."""
    L, c = copes.load(), cache(copes)
    ws, pool, table, length, refs = L.copes_cache_workspace_bytes(c), GOOD["pool"], GOOD["table"], GOOD["length"], GOOD["refs"]
    pool_end, books = pool + 8 * 2 * 2 * 2 * 16 * 64 * 2, (table + 4 * 19, length + 4 * 3, refs + 4 * 7)

    def check(name, call, fine, bad):
        """`bad`: by the number of an argument what makes the call overlap; `fine` does not."""
        for at, values in bad.items():
            for v in values:
                args = list(fine)
                args[at] = v
                refused(copes, call(*args), -1, name)

    check("copes_cache_grow", lambda slots, add, work: L.copes_cache_grow(c, slots, 2, add, 0, work, BIG, None), (0x100, 0x200, WS),
          {0: (*books, table - 4, WS, WS + ws - 4, pool), 1: (*books, length, WS - 4, pool_end - 4),
           2: (pool, pool_end - 16, pool - 16, table, table - 16, 0xA000000, 0xB000010, 0xB000000 - 16)})
    check("copes_cache_fork", lambda a, b, work: L.copes_cache_fork(c, a, b, 2, work, BIG, None), (0x100, 0x200, WS),
          {0: (*books, WS, pool), 1: (*books, WS + ws - 4, pool_end - 4), 2: (pool, pool_end - 16, table, length - 16, refs)})
    check("copes_cache_free", lambda slots: L.copes_cache_free(c, slots, 2, None), (0x100,), {0: (*books, table - 4)})
    check("copes_cache_compact", lambda counts, work: L.copes_cache_compact(c, counts, work, BIG, None), (0x100, WS),
          {0: (*books, pool, pool_end - 4, WS, WS + ws - 4, WS - 4), 1: (pool, pool_end - 16, table, length, refs)})
    check("copes_cache_copy_pages", lambda a, b: L.copes_cache_copy_pages(c, a, b, 2, None), (0x100, 0x200),
          {0: (pool, pool_end - 4, pool - 4), 1: (pool, pool_end - 4)})
    check("copes_cache_append", lambda s, p: L.copes_cache_append(c, 0, s, p, 2, 0x100, 128, 64, 0x100, 128, 64, None),
          (0x100, None), {0: (pool, pool_end - 4), 1: (pool - 4, pool_end - 4)})
    need, out, lse, q = L.copes_paged_attention_workspace_bytes(c, 2, 8), 0xE0000000, 0xE1000000, 0xE2000000

    def attend(slots, q, out, lse, work):
        return L.copes_paged_attention(c, 0, slots, 2, q, 512, 64, 8, 0.1, out, lse, work, 1 << 20, None)

    assert need < 1 << 20
    check("copes_paged_attention", attend, (0x100, q, out, lse, WS),
          {0: (out, out + 2044, lse, lse - 4, WS, WS + need - 4), 1: (WS, WS + need - 2, WS - 2046),
           2: (table, table + 64, length, refs, refs - 16, WS, WS + (need - 1) // 16 * 16, pool),
           3: (*books, WS, WS + need - 4, WS - 60, pool), 4: (pool, pool_end - 16, table, length, refs, out, lse, q)})
    # what is only read may lie anywhere among what is only read: no refusal before the workspace's
    assert L.copes_paged_attention(c, 0, table, 2, q, 512, 64, 8, 0.1, out, lse, None, 0, None) == -4


def test_log_probabilities_into_one_another_or_the_targets_are_refused(copes):
    L = copes.load()
    fine = dict(logits=0x100000, target=0x1000, lp=0x2000, ent=0x3000, ids=0x4000, tlp=0x5000)

    def call(logits, target, lp, ent, ids, tlp):
        return L.copes_token_logprobs(logits, 0, 3, 100, 200, target, 1.0, 5, lp, ent, ids, tlp, None)

    size = dict(logits=1000, target=24, lp=12, ent=12, ids=120, tlp=60)
    for out in ("lp", "ent", "ids", "tlp"):
        for other in set(fine) - {out}:
            step = 8 if out == "ids" else 4
            for at in (fine[other], fine[other] + size[other] - step, fine[other] - size[out] + step):
                refused(copes, call(**{**fine, out: at // step * step}), -1, "copes_token_logprobs")


def test_an_attention_scale_past_fp32_in_log2_is_refused(copes):
    """A score of 0 would be 0 times infinity."""
    L, c = copes.load(), cache(copes)
    for scale, code in [(2.4e38, -1), (-3.4e38, -1), (2.3e38, -4), (-2.3e38, -4)]:  # -4: past this check, no workspace
        refused(copes, L.copes_paged_attention(c, 0, None, 1, 0x100, 256, 64, 4, scale, 0xD000000, None, None, 0, None),
                code, "copes_paged_attention")


def test_workspaces_that_calls_were_given_stay_with_the_handle(copes):
    """A captured call goes on writing to the address that it was given.  (On a handle without its
    constructor, which wants a GPU's tensors.)"""
    c = object.__new__(copes.KVCache)
    c.pool, c.attend_workspace, c._attend_room, c._attend_before, c._streams = torch.empty(0), None, 0, [], {}
    c._attend_shapes = lambda n, q_heads: (1000 * n, None, None)
    given = [(c.attend_space(n, 1), weakref.ref(c.attend_workspace)) for n in (1, 3, 2, 4, 300)]
    gc.collect()
    for (at, size), ws in given:
        assert ws() is not None and ws().data_ptr() == at and ws().numel() == size
    assert [size for (_, size), _ in given] == [1000, 3000, 3000, 6000, 300000]


def test_every_array_of_a_handle_is_noted_on_every_stream_of_its_calls(copes, monkeypatch):
    """On stand-ins for tensors and streams: what is freed later waits for these streams."""
    class Tensor:
        def __init__(self, *streams):
            self.on = [s.cuda_stream for s in streams]

        def record_stream(self, stream):
            self.on.append(stream.cuda_stream)

        def data_ptr(self):
            return 256

    monkeypatch.setattr(copes, "_empty", lambda template, stream: Tensor(stream))
    c = object.__new__(copes.KVCache)
    arrays = [Tensor() for _ in range(5)]
    c.pool, c.table, c.length, c.refs, c.workspace = arrays
    c.pool.device = "cpu"
    c.attend_workspace, c._attend_room, c._attend_before, c._streams = None, 0, [], {}
    c._attend_shapes = lambda n, q_heads: (n, None, None)
    streams = [SimpleNamespace(cuda_stream=i) for i in (5, 9)]
    for n in (1, 10):
        for s in streams:
            c.attend_space(n, 1, s)
            assert c._stream(s) == s.cuda_stream
    for t in arrays + c._attend_before + [c.attend_workspace]:
        assert sorted(set(t.on)) == [5, 9]  # allocated there or noted


def test_the_model_of_the_pages():
    """The bookkeeping that the GPU tests compare with, on a small case by hand."""
    m = model.CacheModel(n_pages=6, page_size=4, n_slots=4, width=3)
    assert m.grow([2, 0], [5, 1]) == 0
    assert m.pages == [[2], [], [0, 1], []] and m.refs == [1, 1, 1, 0, 0, 0]
    assert m.fork([2, 2], [1, 3]) == 0
    assert m.pages == [[2], [0, 3], [0, 1], [0, 4]] and m.copies == [(1, 3), (1, 4)] and m.refs == [3, 1, 1, 1, 1, 0]
    assert m.grow([0, 1], [8, 4]) == 64 and m.grow([0], [12]) == 32 and m.fork([0], [1]) == 32
    assert m.free([2, 2, 9]) == 32 and m.refs == [2, 0, 1, 1, 1, 0]
    assert m.compact() == (4, 1) and m.pages == [[2], [0, 3], [], [0, 1]] and m.refs == [2, 1, 1, 1, 0, 0]
