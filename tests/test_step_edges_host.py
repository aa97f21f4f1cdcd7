"""Calls at the edges of a generating step that the host decides: pools of another form, weights of another type than
the cache, cuts that fp32 rounds away, and what a decoder leaves in a cache where a step fails."""
import glob
import os
import re

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
