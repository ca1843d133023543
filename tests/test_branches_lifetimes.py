"""What a NewTokens of drafted tokens and a PagePool on a stream of their own read is
made known to that stream, and only then."""
from contextlib import nullcontext

import pytest
import torch

from paper_2609_39358_amd import pipeline
from paper_2609_39358_amd import taliesin as T
from paper_2609_39358_amd.device import PagedCache


@pytest.fixture
def calls(monkeypatch):
    """(arrays made known to a stream, a caller's stream, another one); no library call runs."""
    known = []
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda x, s: known.append((x.data_ptr(), s)))
    caller, own = object(), object()
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: caller)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: nullcontext())
    monkeypatch.setattr(pipeline, "_on", lambda s: nullcontext())
    monkeypatch.setattr(T, "_fits", lambda *a: None)
    for name in ("tl_keep", "tl_pages_take", "tl_pages_fork", "tl_pages_free"):
        monkeypatch.setattr(T, name, lambda *a, **k: None)
    return known, own


def words(*shape, dtype=torch.int32):
    return torch.zeros(shape, dtype=dtype)


@pytest.mark.parametrize("own_stream", [False, True])
def test_drafted_tokens(calls, own_stream):
    known, own = calls
    ctx = T.tl_ctx_create(b"tenant", b"model", 1, 2, 64, "bf16", 16)
    cache = PagedCache(1, 4, ctx.slab_bytes, "cpu")
    arrays = [words(3), words(2), words(1, 2, 4), torch.zeros(8, 32, 2)]
    tree = [words(2, 1, dtype=torch.int64), words(2)]
    t = pipeline.NewTokens(ctx, cache, 4, 2, *arrays, own if own_stream else None, *tree)
    kept = [words(2), words(2)]
    t.keep(*kept)
    want = {(x.data_ptr(), own) for x in arrays + tree + kept} if own_stream else set()
    assert set(known) == want


@pytest.mark.parametrize("own_stream", [False, True])
def test_pools(calls, own_stream):
    known, own = calls
    ctx = T.tl_ctx_create(b"tenant", b"model", 1, 2, 64, "bf16", 16)
    pool = pipeline.PagePool(ctx, PagedCache(1, 4, ctx.slab_bytes, "cpu"), used=[2], stream=own if own_stream else None)
    assert pool.refs.tolist() == [[0, 0, 1, 0]]
    have, want_, tables, parent, first = words(2), words(2), words(1, 2, 4), words(3), words(2)
    pool.take(have, want_, tables)
    out, lens = pool.fork(have, tables, parent)
    assert out.shape == (1, 3, 4) and lens.shape == (3,) and pool.status.shape == (3,)
    pool.free(tables, first)
    want = {(x.data_ptr(), own) for x in (have, want_, tables, parent, first)} if own_stream else set()
    assert set(known) == want
