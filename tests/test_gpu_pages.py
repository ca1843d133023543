"""tl_pages_copy, tl_pages_fork, tl_pages_take and tl_pages_free against host
arithmetic: every byte of every layer, every table entry, every page's count; over
element types, page sizes, groups of layers, pages that are missing, pools that run
out; captured and replayed."""
import numpy as np
import pytest
import torch

from paper_2609_39358_amd import taliesin as T
from tests import pages_case as hc
from tests.pages_case import DEV, Pages, up

pytestmark = pytest.mark.gpu

SHAPES = [  # P, H, D, cache, layers, group_of, pad
    (16, 4, 64, "fp8_scaled", 3, None, 0),
    (16, 8, 128, "bf16", 2, [0, 1], 0),
    (104, 1, 64, "fp8_scaled", 2, [1, 0], 16),
    (7, 16, 64, "bf16", 2, None, 0),
    (256, 2, 256, "fp8_scaled", 1, None, 1024),
    (1, 8, 128, "bf16", 2, [0, 2], 0),
    (16, 2, 64, "f32", 2, None, 0),
    (64, 3, 16, "fp8", 3, None, 0),  # rows of 48 bytes
    (1024, 1, 5, "fp8", 2, None, 0),  # rows of 5 bytes
    (48, 7, 64, "fp8_scaled", 40, [l % 3 for l in range(40)], 0),
]


def stream():
    return torch.cuda.current_stream()


@pytest.mark.parametrize("P,H,D,cache,layers,group_of,pad", SHAPES)
@pytest.mark.parametrize("whole", [True, False])
def test_copy(P, H, D, cache, layers, group_of, pad, whole):
    c = Pages(3, P, H, D, cache, 23, layers, group_of, pad).up()
    n = 9
    ids = np.stack([c.r.permutation(c.n_pages)[:2 * n] for _ in range(c.groups)]).astype(np.int32)
    src, dst = ids[:, :n].copy(), ids[:, n:].copy()
    src[0, 2], dst[c.groups - 1, 3], src[0, 4] = -1, -1, c.n_pages  # not in that group
    src[:, 5] = src[:, 6]  # one page to two
    rows = None if whole else np.array([0, 1, P, P, max(1, P // 2), P + 7, (P + 1) // 2, P - 1, 2 ** 32 - 1], np.int64)
    d = [up(src), up(dst), None if whole else up(rows.astype(np.uint32).view(np.int32))]
    T.tl_pages_copy(c.ctx, stream(), c.paged.tl(), n, *d)
    hc.copy(c, src, dst, rows)
    torch.cuda.synchronize()
    c.same()


def a_pool(c, n_parents, width, kv_len, shared, reserve):
    """Parents whose first `shared` pages are one and the same, their counts and
    tables; `reserve` pages are left free, in between."""
    G = c.groups
    refs, tables = np.zeros((G, c.n_pages), np.int32), np.full((G, n_parents, width), -1, np.int32)
    for g in range(G):
        ids = list(c.r.permutation(c.n_pages))
        common = [ids.pop() for _ in range(shared)]
        for i, k in enumerate(kv_len):
            m = -(-int(k) // c.P)
            mine = (common + [ids.pop() for _ in range(max(0, m - shared))])[:m]
            tables[g, i, :m] = mine
            for p in mine:
                refs[g, p] += 1
        while len(ids) > reserve:  # others'
            refs[g, ids.pop()] += 1 + int(c.r.integers(3))
    return refs, tables


def fork_on_device(c, pool, d_kv, d_tables, n_parents, parent, width, ws=None):
    n = len(parent)
    out = torch.full((c.groups, n, width), 77, dtype=torch.int32, device=DEV)
    lens, status = torch.full((n,), 77, dtype=torch.int32, device=DEV), torch.zeros(n, dtype=torch.uint8, device=DEV)
    size = T.tl_pages_workspace_bytes(c.ctx, n, c.n_pages)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV)
    T.tl_pages_fork(c.ctx, stream(), pool, c.paged.tl(), n_parents, d_kv, d_tables, n, up(parent), lens, out, width, ws, size, status)
    return out, lens, status


def equal(got, want, what):
    got = got.cpu().numpy().astype(np.int64)
    want = np.asarray(want).astype(np.int64)
    assert np.array_equal(got, want), (what, np.argwhere(got != want)[:5])


@pytest.mark.parametrize("P,H,D,cache,layers,group_of,pad", SHAPES)
@pytest.mark.parametrize("reserve", [40, 3, 0])
def test_fork_take_free(P, H, D, cache, layers, group_of, pad, reserve):
    c = Pages(4, P, H, D, cache, 90, layers, group_of, pad).up()
    kv = np.array([3 * P + (P > 1), 2 * P, 0, 1, 5 * P - 1, 4 * P], np.int64)
    width = 8
    refs, tables = a_pool(c, len(kv), width, kv, 2, reserve)
    tables[0, 0, 1] = -1  # a page that was not restored
    tables[c.groups - 1, 4, 4] = -1  # the last one
    kv[5] = width * P + 1  # longer than its row
    parent = np.array([0, 0, 4, 1, 2, 3, 3, -1, 4, 5, 6, 0, 2 ** 31 - 1, 1, 3], np.int64)
    d_refs, d_tables, d_kv = up(refs), up(tables), up(kv)
    pool = T.make_pool(d_refs)
    out, lens, status = fork_on_device(c, pool, d_kv, d_tables, len(kv), parent, width)
    t, n, s = hc.fork(c, refs, kv, tables, parent)
    if reserve == 40:
        assert (s == T.ACCEPT).sum() == 11
    torch.cuda.synchronize()
    equal(status, s, "status")
    equal(lens, n, "lengths")
    equal(out, t, "tables")
    equal(d_refs, refs, "counts")
    c.same("fork")
    # room for more: none, a few tokens, whole pages, too many
    have = n.copy()
    want = have + np.array([0, 1, P, 3 * P, 0, P + 1, 2 * P, 5, 1, P, 0, 7 * P, width * P + 1, 1, 2])
    want[4] = 0
    size = T.tl_pages_workspace_bytes(c.ctx, len(parent), c.n_pages)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    T.tl_pages_take(c.ctx, stream(), pool, len(parent), up(have), up(want), out, width, ws, size, status)
    s = hc.take(c, refs, have, want, t)
    torch.cuda.synchronize()
    equal(status, s, "status")
    equal(out, t, "tables")
    equal(d_refs, refs, "counts")
    # what lies wholly behind and before some tokens is given back, then everything
    first = np.minimum(have, 2 ** 31 - 1)
    end = np.array([0, P, P - 1, 2 * P, 1, 99 * P, P + 1, 0, 3 * P, P, 2 * P, P, 0, 4 * P, 2 ** 32 - 1], np.int64)
    for a, b in ((first, None), (None, end), (end, first), (None, None)):
        dev = [None if x is None else up(x.astype(np.uint32).view(np.int32)) for x in (a, b)]
        T.tl_pages_free(c.ctx, stream(), pool, len(parent), out, width, *dev)
        hc.give_back(c, refs, t, a, b)
        torch.cuda.synchronize()
        equal(out, t, "tables")
        equal(d_refs, refs, "counts")
    assert (t == -1).all()
    c.same("all")


@pytest.mark.parametrize("n_pages", [1, 5000, 70001])
def test_large_pools_and_many_requests(n_pages):
    """Free pages far apart, more requests than the planning workgroup has threads, and ranges of
    all lengths."""
    c = Pages(5, 16, 1, 64, "fp8", 1, 1).up()
    c.n_pages = n_pages
    r = np.random.default_rng(6)
    refs = (r.random((1, n_pages)) < 0.7).astype(np.int32) * r.integers(1, 5, (1, n_pages)).astype(np.int32)
    refs[0, r.integers(0, n_pages, 50 if n_pages > 1 else 0)] = -1  # given back once too often: free
    refs[0, :n_pages // 3] = 1
    n, width = 3001, 70
    have = r.integers(0, 16 * 30, n)
    want = have + np.where(r.random(n) < 0.05, r.integers(0, 16 * 40, n), r.integers(0, 20, n))
    tables = np.full((1, n, width), -1, np.int32)
    tables[0, r.integers(0, n, 500), r.integers(0, width, 500)] = 0
    d_refs, d_tables = up(refs), up(tables)
    size = T.tl_pages_workspace_bytes(c.ctx, n, n_pages)
    ws, status = torch.empty(size, dtype=torch.uint8, device=DEV), torch.empty(n, dtype=torch.uint8, device=DEV)
    T.tl_pages_take(c.ctx, stream(), T.make_pool(d_refs), n, up(have), up(want), d_tables, width, ws, size, status)
    s = hc.take(c, refs, have, want, tables)
    torch.cuda.synchronize()
    assert n_pages == 70001 or (s == T.MISSING).any()
    equal(status, s, "status")
    equal(d_tables, tables, "tables")
    equal(d_refs, refs, "counts")


def test_captured():
    """A step of branches, captured and replayed with other parents and lengths, eager work between."""
    P, width = 16, 6
    c = Pages(7, P, 4, 64, "fp8_scaled", 64, 2).up()
    kv = np.array([20, 35, 64, 7], np.int64)
    refs, tables = a_pool(c, len(kv), width, kv, 0, 40)
    d_refs, d_tables, d_kv = up(refs), up(tables), up(kv)
    n = 5
    pool, d_parent = T.make_pool(d_refs), up(np.zeros(n))
    out = torch.full((1, n, width), -1, dtype=torch.int32, device=DEV)
    lens, want, status = (torch.zeros(n, dtype=torch.int32, device=DEV) for _ in range(3))
    size = T.tl_pages_workspace_bytes(c.ctx, n, c.n_pages)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV)
    cache = c.paged.tl()

    def step():
        T.tl_pages_free(c.ctx, stream(), pool, n, out, width)
        T.tl_pages_fork(c.ctx, stream(), pool, cache, len(kv), d_kv, d_tables, n, d_parent, lens, out, width, ws, size)
        torch.add(lens, 9, out=want)
        T.tl_pages_take(c.ctx, stream(), pool, n, lens, want, out, width, ws, size)

    t = np.full((1, n, width), -1, np.int32)

    def on_host(parent):
        hc.give_back(c, refs, t)
        new, k, _ = hc.fork(c, refs, kv, tables, parent)
        t[:] = new
        hc.take(c, refs, k, k + 9, t)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    on_host([0] * n)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(4):
        r = np.random.default_rng(seed)
        parent = r.integers(0, len(kv), n)
        kv[:] = np.minimum(r.integers(0, 64, len(kv)), np.array([32, 48, 64, 16]))
        d_parent.copy_(up(parent))
        d_kv.copy_(up(kv))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        on_host(parent)
        equal(out, t, "tables")
        equal(d_refs, refs, "counts")
        c.same("replay %d" % seed)


def test_offsets_past_32_bits():
    """Pages beyond the first 4 GiB of a cache, copied and branched."""
    from paper_2609_39358_amd.device import PagedCache

    c = Pages(8, 16, 8, 128, "fp8_scaled", 12, 1).up()
    n_pages = (9 << 29) // c.stride
    far = n_pages - c.n_pages
    big = [torch.empty((n_pages, c.stride), dtype=torch.uint8, device=DEV) for _ in range(2)]
    for b, x in zip(big, c.dev):
        b[far:] = x
    paged = PagedCache(1, n_pages, c.stride, DEV, [big[0]], [big[1]])
    src, dst, rows = np.array([[0, 5]]), np.array([[9, 2]]), np.array([16, 7])
    T.tl_pages_copy(c.ctx, stream(), paged.tl(), 2, up(src + far), up(dst + far), up(rows))
    hc.copy(c, src, dst, rows)
    refs = np.ones((1, n_pages), np.int32)
    refs[0, far + 10] = 0
    tables = np.array([[[far + 1, far + 4, -1]]])
    size = T.tl_pages_workspace_bytes(c.ctx, 1, n_pages)
    out, lens = torch.zeros((1, 1, 3), dtype=torch.int32, device=DEV), up(np.zeros(1))
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    d_refs = up(refs)
    T.tl_pages_fork(c.ctx, stream(), T.make_pool(d_refs), paged.tl(), 1, up(np.array([27])), up(tables), 1, up(np.zeros(1)), lens, out, 3, ws, size)
    hc.copy(c, np.array([[4]]), np.array([[10]]), [11])
    torch.cuda.synchronize()
    assert out.tolist() == [[[far + 1, far + 10, -1]]] and lens.tolist() == [27]
    assert d_refs[0, far + 1].item() == 2 and d_refs[0, far + 10].item() == 1
    c.dev = torch.stack([b[far:] for b in big])
    c.same()


def test_copies_captured():
    c = Pages(9, 16, 4, 64, "bf16", 40, 3).up()
    src, dst, rows = (up(np.zeros((1, 6))) for _ in range(3))
    cache = c.paged.tl()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        T.tl_pages_copy(c.ctx, side, cache, 6, src, dst, rows)
    for turn in range(3):
        ids = c.r.permutation(40)[:12]
        n = c.r.integers(0, 17, 6)
        for x, y in ((src, ids[:6]), (dst, ids[6:]), (rows, n)):
            x.copy_(up(y[None]))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        hc.copy(c, ids[None, :6], ids[None, 6:], n)
        c.same("replay %d" % turn)
