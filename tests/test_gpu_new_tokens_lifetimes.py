"""A step on a stream of its own whose arrays are dropped at once: the caller's
stream, which reuses freed memory, does not get theirs while the step waits."""
import numpy as np
import pytest
import torch

from paper_2609_39358_amd import taliesin as T
from paper_2609_39358_amd.device import PagedCache
from paper_2609_39358_amd.pipeline import NewTokens

pytestmark = pytest.mark.gpu

DEV = "cuda"


def test_arrays_that_are_dropped_while_the_stream_waits():
    H, HQ, D, P, kv = 2, 4, 64, 16, 300
    ctx = T.tl_ctx_create(b"tenant", b"model", 1, H, D, "bf16", P)
    n_pages = -(-kv // P)
    cache = PagedCache(1, n_pages, ctx.slab_bytes, DEV)
    for x in cache.k + cache.v:
        x.view(torch.bfloat16).normal_()
    before = [x.clone() for x in cache.k + cache.v]
    a = np.arange(512)[:, None] * 100.0 ** (-np.arange(D // 2) / (D // 2))
    host = [np.array([0, 1], np.int32), np.array([kv], np.int32), np.random.default_rng(0).permutation(n_pages).astype(np.int32)[None, None],
            np.stack([np.cos(a), np.sin(a)], -1).astype(np.float32)]
    qkv = torch.randn((1, HQ + 2 * H, D), device=DEV).to(torch.bfloat16)

    def step(stream, wait):
        arrays = [torch.from_numpy(x).to(DEV) for x in host]
        torch.cuda.synchronize()
        at = {x.data_ptr() for x in arrays}
        if wait:
            with torch.cuda.stream(stream):
                torch.cuda._sleep(20_000_000)  # cycles: some milliseconds
        t = NewTokens(ctx, cache, HQ, 1, *arrays, stream=stream)
        q, k, v = qkv.split([HQ, H, H], dim=1)
        return t.layer(0, q, k, v), at

    want, _ = step(None, False)
    torch.cuda.synchronize()
    for x, y in zip(cache.k + cache.v, before):
        x.copy_(y)
    side = torch.cuda.Stream()
    got, at = step(side, True)
    fresh = [torch.full_like(torch.from_numpy(x), 0, device=DEV) for x in host * 4]  # on the caller's stream
    if not side.query():  # still waiting, so the arrays are not read yet
        assert not at & {x.data_ptr() for x in fresh}
    torch.cuda.synchronize()
    assert torch.equal(got.view(torch.int16), want.view(torch.int16))
