"""Refusals of a generating step's C entries: every case fails its checks before any CUDA call, with a message that
names the entry; the fake addresses are never read."""
import copy
import ctypes
import os

import pytest
import torch

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def copes():
    from paper_2608_02391_gb300 import build, copes as c
    if not os.path.exists(c.LIB_PATH):
        build.build()
    c.load()
    return c


def refused(copes, rc, code, name):
    assert rc == code, (name, rc, copes.last_error())
    assert name in copes.last_error()


def test_drawing_is_refused(copes):
    fine = dict(logits=0x100000, dtype=0, n=3, vocab=100, row=200, u=0x1000, scale=1.0, top_k=5, top_p=0.9, min_p=0.1, ids=0x2000,
                lp=0x3000, kept=0x4000)
    call = lambda **kw: copes.load().copes_sample_tokens(*{**fine, **kw}.values(), None)
    for kw, code in [(dict(dtype=2), -1), (dict(dtype=3), -1), (dict(n=-1), -1), (dict(vocab=0), -1), (dict(vocab=4_000_001), -3),
                     (dict(n=(1 << 27) + 1), -3), (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=NAN), -1), (dict(scale=INF), -1),
                     (dict(scale=1e-31), -1), (dict(top_k=-1), -1), (dict(top_p=0.0), -1), (dict(top_p=1.01), -1), (dict(top_p=NAN), -1),
                     (dict(min_p=-0.1), -1), (dict(min_p=1.1), -1), (dict(min_p=NAN), -1), (dict(logits=None), -1), (dict(u=None), -1),
                     (dict(ids=None), -1), (dict(lp=None), -1), (dict(kept=None), -1), (dict(logits=0x100001), -2), (dict(u=0x1002), -2),
                     (dict(ids=0x2004), -2), (dict(lp=0x3001), -2), (dict(kept=0x4002), -2), (dict(dtype=1, logits=0x100002), -2)]:
        refused(copes, call(**kw), code, "copes_sample_tokens")
    size = dict(logits=1000, u=12, ids=24, lp=12, kept=12)
    for out in ("ids", "lp", "kept"):
        step = 8 if out == "ids" else 4
        for other in set(size) - {out}:
            for at in (fine[other], fine[other] + size[other] - step, fine[other] - size[out] + step):
                refused(copes, call(**{out: at // step * step}), -1, "copes_sample_tokens")


def test_norms_are_refused(copes):
    fine = dict(dtype=0, n=3, hidden=64, x=0x10000, x_row=64, y=0x20000, y_row=64, ow=0x30000, gate=0x40000, gate_row=64, scale=1.0,
                w=0x50000, eps=1e-6, s=0x60000, s_row=64, h=0x70000, h_row=64)
    call = lambda **kw: copes.load().copes_residual_norm(*{**fine, **kw}.values(), None)
    for kw, code in [(dict(dtype=2), -1), (dict(dtype=3), -1), (dict(n=-1), -1), (dict(hidden=0), -1), (dict(hidden=(1 << 24) + 1), -3),
                     (dict(x=None), -1), (dict(y=None), -1), (dict(y=None, s=None, ow=None), -1), (dict(y=None, s=None, gate=None), -1),
                     (dict(s=None, h=None, w=None), -1), (dict(w=None), -1), (dict(h=None), -1), (dict(eps=0.0), -1), (dict(eps=NAN), -1),
                     (dict(eps=INF), -1), (dict(eps=-1e-6), -1), (dict(scale=NAN), -1), (dict(scale=INF), -1), (dict(x_row=-64), -1),
                     (dict(gate_row=-1), -1), (dict(s_row=63), -1), (dict(h_row=0), -1), (dict(y_row=1 << 41), -1), (dict(x=0x10001), -2),
                     (dict(y=0x20001), -2), (dict(ow=0x30001), -2), (dict(gate=0x40001), -2), (dict(w=0x50001), -2), (dict(s=0x60001), -2),
                     (dict(h=0x70001), -2), (dict(dtype=1, x=0x10002), -2)]:
        refused(copes, call(**kw), code, "copes_residual_norm")
    for out in ("s", "h"):
        for other in ("x", "y", "gate", "ow", "w", "s", "h"):
            size = 128 if other in ("ow", "w") else 384
            for at in (fine[other] + size - 2, fine[other] - 382) + (() if (out, other) in (("s", "x"), ("h", "y")) else (fine[other],)):
                if out != other:
                    refused(copes, call(**{out: at}), -1, "copes_residual_norm")
    refused(copes, call(s=0x10000, s_row=65), -1, "copes_residual_norm")  # in place, but of other rows
    refused(copes, call(h=0x20000, h_row=128), -1, "copes_residual_norm")


CACHE = dict(pool=0x1000000, dtype=3, n_pages=8, n_layers=2, n_kv_heads=2, page_size=16, head_dim=64, table=0x9000000, n_slots=4,
             table_width=5, length=0xA000000, refs=0xB000000)


def cache(copes, **kw):
    f = {**CACHE, **kw}
    return ctypes.byref(copes.KVCacheDesc(*[f[name] for name, _ in copes.KVCacheDesc._fields_]))


def test_8_bit_caches_are_refused(copes):
    L = copes.load()
    for kw, code in [(dict(head_dim=8), -3), (dict(head_dim=72), -3), (dict(head_dim=272), -3), (dict(dtype=2), -1), (dict(dtype=4), -1),
                     (dict(pool=0x1000008), -2), (dict(page_size=0), -1)]:
        c = cache(copes, **kw)
        refused(copes, L.copes_cache_append(c, 0, 0x100, None, 1, 0x200, 64, 64, 0x400, 64, 64, None), code, "copes_cache_append")
        refused(copes, L.copes_cache_read(c, 0, 0x100, None, 1, 0x1000, 128, 64, 0x2000, 128, 64, None), code, "copes_cache_read")
        assert L.copes_cache_workspace_bytes(c) == 0 and L.copes_paged_attention_workspace_bytes(c, 1, 4) == 0
    layer = 2 * 2 * 16 * 65  # codes, and a byte for each key and value of a head
    assert copes.KVCache.layer_bytes(2, 16, 64) == layer and copes.KVCache.layer_bytes(1, 1, 16) == 48
    end = 0x1000000 + 8 * 2 * layer
    c = cache(copes)
    for k in (0x1000000, end - 2, 0x1000000 - 254):
        refused(copes, L.copes_cache_append(c, 0, 0x100, None, 1, k, 128, 64, 0x400, 128, 64, None), -1, "copes_cache_append")
    refused(copes, L.copes_cache_append(c, 0, 0x100, None, 1, 0x201, 128, 64, 0x400, 128, 64, None), -2, "copes_cache_append")
    need = L.copes_paged_attention_workspace_bytes(c, 2, 8)
    attend = lambda q, out, lse: L.copes_paged_attention(c, 0, None, 2, q, 512, 64, 8, 0.1, out, lse, 0xC000000, need, None)
    for q, out, lse, code in [(0x101, 0xD000000, None, -2), (0xD000000 + 2046, 0xD000000, None, -1), (0x100, 0xD000000, 0xD000000 + 2044, -1),
                              (0x100, end - 16, None, -1)]:
        refused(copes, attend(q, out, lse), code, "copes_paged_attention")


def test_reading_back_is_refused(copes):
    L, c = copes.load(), cache(copes, dtype=0)
    pool_end = 0x1000000 + 8 * 2 * 2 * 2 * 16 * 64 * 2
    fine = dict(layer=0, slots=0x100, position=0x200, n=3, k=0x10000, k_row=128, k_head=64, v=0x20000, v_row=128, v_head=64)
    call = lambda **kw: L.copes_cache_read(c, *{**fine, **kw}.values(), None)
    for kw, code in [(dict(layer=2), -1), (dict(layer=-1), -1), (dict(slots=0x102), -2), (dict(position=0x201), -2), (dict(n=-1), -1),
                     (dict(slots=None, n=5), -3), (dict(k=None), -1), (dict(v=None), -1), (dict(k=0x10001), -2), (dict(v=0x20001), -2),
                     (dict(k_row=-128), -1), (dict(v_head=-64), -1), (dict(k_row=1 << 41), -1), (dict(k_head=63), -1), (dict(v_row=127), -1),
                     (dict(k_row=64, k_head=128), -1), (dict(k=0x20000), -1), (dict(k=0x20000 - 766), -1), (dict(v=0x1000000), -1),
                     (dict(k=pool_end - 2), -1), (dict(k=0x100), -1), (dict(v=0x200), -1), (dict(k=0x9000000), -1), (dict(v=0xA000000), -1),
                     (dict(v=0xB000000 - 766), -1)]:
        refused(copes, call(**kw), code, "copes_cache_read")
    refused(copes, L.copes_cache_read(None, *fine.values(), None), -1, "copes_cache_read")


def test_the_binding_refuses_other_shapes_and_types(copes):
    x, w = torch.zeros(3, 8), torch.zeros(8)
    with pytest.raises(AssertionError):
        copes.residual_norm(x, w)  # not on a GPU
    with pytest.raises(AssertionError):
        copes.sample_tokens(x, torch.zeros(3))
    with pytest.raises(AssertionError):
        copes.KVCache(torch.zeros(4, 2, 100, dtype=torch.uint8), torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32),
                      torch.zeros(4, dtype=torch.int32), heads=(1, 1, 16))
