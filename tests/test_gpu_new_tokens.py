"""A prompt's KV is appended, saved, damaged, restored and continued: records of
appended pages are the oracle's byte for byte, and what a request answers on
restored pages has the bits of what it answers on the pages that were saved."""
import numpy as np
import pytest
import torch

import workloads as wl
from oracle import taliesin_ref as ref
from paper_2609_39358_amd import taliesin as T
from paper_2609_39358_amd.device import PagedCache
from paper_2609_39358_amd.pipeline import NewTokens, RestorePipeline, Store

pytestmark = pytest.mark.gpu

DEV = "cuda"
L, H, HQ, P = 2, 4, 8, 16


def up(a, dt=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a).astype(dt, copy=False)).to(DEV)


def angles(n, D):
    a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(D // 2) / (D // 2))
    return up(np.stack([np.cos(a), np.sin(a)], -1), np.float32)


def step(ctx, cache, table, kv_len, new, qkv, cos_sin, stream=None):
    """One request's new tokens through every layer; their results and lse."""
    t = NewTokens(ctx, cache, HQ, new, up([0, new]), up([kv_len]), up(table[None, None, :]), cos_sin, stream)
    outs, lses = [], []
    for l in range(L):
        lse = torch.empty((new, HQ), dtype=torch.float32, device=DEV)
        q, k, v = qkv[l].split([HQ, H, H], dim=1)
        outs.append(t.layer(l, q, k, v, lse))
        lses.append(lse)
    torch.cuda.synchronize()
    assert bool((t.status == T.ACCEPT).all())
    return outs, lses


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("D", [64, 128])
def test_save_restore_and_go_on(cache, D):
    n, tail, more = 37, 9, 3  # whole blocks, the tokens behind them, decode steps
    dtype = {"bf16": 1, "fp8_scaled": 5}[cache]
    lay = ref.Layout(L, H, D, dtype, P)
    ns = ref.namespace_digest(b"tenant", b"model", lay)
    ctx = T.tl_ctx_create(b"tenant", b"model", L, H, D, cache, P)
    assert ctx.slab_bytes == lay.slab_bytes and ctx.record_bytes == lay.record_bytes
    total = n * P + tail + more
    g = torch.Generator(device=DEV).manual_seed(5)
    qkv = torch.randn((L, total, HQ + 2 * H, D), dtype=torch.float32, device=DEV, generator=g).to(torch.bfloat16)
    cos_sin = angles(total, D)
    prompt = wl.tokens(n * P + tail, 3)

    # the first time: prefill, then the tail and decode
    pages = np.random.default_rng(1).permutation(64)[:n + 1].astype(np.int32)
    kv = PagedCache(L, 64, ctx.slab_bytes, DEV).zero_()
    at = [n * P, n * P + tail] + [n * P + tail + i + 1 for i in range(more)]
    step(ctx, kv, pages, at[0], at[0], qkv[:, :at[0]], cos_sin)

    # its blocks are saved
    keys = T.tl_block_keys(ctx, prompt)
    toks = prompt[:n * P].reshape(n, P)
    assert len(keys) == n
    store = Store(ctx, n)
    T.tl_save(ctx, torch.cuda.current_stream(), n, kv.tl(),
              T.make_blocks(up(keys, np.uint8), torch.arange(n, device=DEV), up(toks.view(np.int32)), up(pages[None, :n])),
              store.records.ptrs)
    store.add(keys, range(n))
    torch.cuda.synchronize()
    hk, hv = ([t.cpu().numpy() for t in x] for x in (kv.k, kv.v))
    recs, _ = ref.save(lay, ns, hk, hv, pages[None, :n], [k.tobytes() for k in keys], np.arange(n), toks)
    got = store.records.buf.cpu().numpy()
    assert all(got[b].tobytes() == recs[b] for b in range(n))

    want = [step(ctx, kv, pages, b, b - a, qkv[:, a:b], cos_sin) for a, b in zip(at, at[1:])]

    # a later request restores them, on a stream of its own, and goes on behind them
    stream = torch.cuda.Stream()
    pool = PagedCache(L, 48, ctx.slab_bytes, DEV).zero_()
    res = RestorePipeline(store, pool, stream).restore([prompt], [0])
    assert res.hits == [n]
    table = np.arange(n + 1, dtype=np.int32)  # restored block i is in page i
    for (a, b), (outs, lses) in zip(zip(at, at[1:]), want):
        o, e = step(ctx, pool, table, b, b - a, qkv[:, a:b], cos_sin, stream)
        for l in range(L):
            assert torch.equal(o[l].view(torch.int16), outs[l].view(torch.int16)), (a, l)
            assert torch.equal(e[l], lses[l]), (a, l)
            assert bool(torch.isfinite(o[l].float()).all())
    assert [int(x) for x in res.verdicts.cpu()] == [ref.ACCEPT] * n
    for l in range(L):
        for x, y in ((pool.k[l], kv.k[l]), (pool.v[l], kv.v[l])):
            assert torch.equal(x[:n + 1], y[torch.from_numpy(pages.astype(np.int64)).to(DEV)])


def test_a_damaged_scale_is_refused():
    """One bit of a page's scale byte is as much a part of the record as its codes."""
    D, n = 64, 6
    lay = ref.Layout(L, H, D, 5, P)
    ns = ref.namespace_digest(b"tenant", b"model", lay)
    ctx = T.tl_ctx_create(b"tenant", b"model", L, H, D, "fp8_scaled", P)
    kv = PagedCache(L, 8, ctx.slab_bytes, DEV).zero_()
    qkv = torch.randn((L, n * P, HQ + 2 * H, D), device=DEV).to(torch.bfloat16)
    pages = np.arange(n, dtype=np.int32)
    step(ctx, kv, pages, n * P, n * P, qkv, None)
    prompt = wl.tokens(n * P, 3)
    keys, toks = T.tl_block_keys(ctx, prompt), prompt.reshape(n, P)
    store = Store(ctx, n)
    T.tl_save(ctx, torch.cuda.current_stream(), n, kv.tl(),
              T.make_blocks(up(keys, np.uint8), torch.arange(n, device=DEV), up(toks.view(np.int32)), up(pages[None])),
              store.records.ptrs)
    store.add(keys, range(n))
    at = lay.payload_offset + P * H * D + 1  # the second head's scale in the record's first slab
    store.records.buf[2, at] ^= 1
    pool = PagedCache(L, n, ctx.slab_bytes, DEV).zero_()
    res = RestorePipeline(store, pool).restore([prompt], [0])
    torch.cuda.synchronize()
    recs = [r.tobytes() for r in store.records.buf.cpu().numpy()]
    dk = [np.zeros((n, lay.slab_bytes), np.uint8) for _ in range(L)]
    dv = [np.zeros((n, lay.slab_bytes), np.uint8) for _ in range(L)]
    want = ref.restore(lay, ns, recs, [k.tobytes() for k in keys], np.arange(n), toks, pages[None], dk, dv)
    assert want[2] != ref.ACCEPT and want.count(ref.ACCEPT) == n - 1
    assert [int(x) for x in res.verdicts.cpu()] == want
    for l in range(L):
        assert np.array_equal(pool.k[l].cpu().numpy(), dk[l]) and np.array_equal(pool.v[l].cpu().numpy(), dv[l])
