"""tl_keep against host arithmetic: every byte of every layer, lengths and statuses,
over page sizes, few and many rows, scales that agree, rise and fall between pages,
and entries that cannot be kept."""
import numpy as np
import pytest
import torch

from paper_2609_39358_amd import taliesin as T
from tests import pages_case as hc
from tests.pages_case import DEV, Pages, up

pytestmark = pytest.mark.gpu


def run(c, tables, new, kv_len, kept, n_keep=None):
    """On the device and on the host; lengths and statuses are compared, then every byte."""
    n, rows = len(new), sum(new)
    off = np.concatenate([[0], np.cumsum(new)])
    flat = np.full(max(rows, 1), 12345, np.int64)
    for i, k in enumerate(kept):
        flat[off[i]:off[i] + len(k)] = k
    count = np.array([len(k) for k in kept]) if n_keep is None else np.array(n_keep)
    d = [up(off), up(np.array(kv_len, np.int64).astype(np.uint32).view(np.int32)), up(tables)]
    batch = T.make_batch(n, rows, *d, tables.shape[2])
    lens, status = torch.full((n,), 77, dtype=torch.int32, device=DEV), torch.zeros(n, dtype=torch.uint8, device=DEV)
    flat = flat.astype(np.uint32).view(np.int32)
    T.tl_keep(c.ctx, torch.cuda.current_stream(), batch, c.paged.tl(), up(count), up(flat), lens, status)
    torch.cuda.synchronize()
    want = hc.keep(c, tables, new, kv_len, kept)
    c.same()
    return [int(x) & 0xFFFFFFFF for x in lens.cpu()], [int(x) for x in status.cpu()], want


def make(seed, P, H, D, cache, new, kv_len, layers=2, group_of=None, pad=0, spread=3):
    width = max(1, max(-(-k // P) for k in kv_len)) + 1
    first = [max(0, (k - a)) // P for a, k in zip(new, kv_len)]
    used = sum(-(-k // P) - f for k, f in zip(kv_len, first))
    c = Pages(seed, P, H, D, cache, used + 2, layers, group_of, pad, spread).up()
    tables = np.full((c.groups, len(new), width), -1, np.int32)  # pages before the new tokens are not there
    for g in range(c.groups):
        ids = list(c.r.permutation(c.n_pages).astype(np.int32))
        for i, k in enumerate(kv_len):
            for j in range(first[i], -(-k // P)):
                tables[g, i, j] = ids.pop()
    return c, tables


def some(r, new, n):
    return sorted(r.choice(new, n, replace=False).tolist())


FEW = [  # P, H, D, layers, group_of, pad
    (16, 4, 64, 3, [0, 1, 0], 0),
    (16, 8, 128, 2, None, 0),
    (104, 1, 64, 2, [1, 0], 16),
    (7, 16, 64, 2, None, 0),
    (256, 3, 256, 1, None, 1024),
    (1, 8, 128, 2, None, 0),
    (32, 6, 256, 2, None, 0),
]


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("P,H,D,layers,group_of,pad", FEW)
@pytest.mark.parametrize("spread", [0, 4])
def test_drafts(cache, P, H, D, layers, group_of, pad, spread):
    r = np.random.default_rng(1)
    new = [8, 1, 64, 33, 5, 0, 48, 21, 64, 40]
    kv_len = [a + h for a, h in zip(new, [0, 15, 16, 31, 100, 3, 7, 250, 1, 17])]
    kept = [[0, 3, 7], [0], some(r, 64, 9), some(r, 33, 33), [], [], some(r, 48, 1), [0, 1, 2], some(r, 64, 40), [0, 1, 2, 39]]
    c, tables = make(2, P, H, D, cache, new, kv_len, layers, group_of, pad, spread)
    lens, status, want = run(c, tables, new, kv_len, kept)
    assert lens == want[0] and status == want[1] and set(status) == {T.ACCEPT}


@pytest.mark.parametrize("cache,requests", [("bf16", 40), ("fp8_scaled", 40), ("fp8_scaled", 66)])
def test_many_slabs(cache, requests):
    """So much work that a wavefront takes several layers, 4 or 8 slabs of them."""
    r = np.random.default_rng(9)
    new = r.integers(1, 12, requests).tolist()
    kv_len = [a + int(h) for a, h in zip(new, r.integers(0, 40, requests))]
    kept = [some(r, n, int(r.integers(0, min(n, 4) + 1))) for n in new]
    c, tables = make(10, 16, 16, 64, cache, new, kv_len, layers=25)
    lens, status, want = run(c, tables, new, kv_len, kept)
    assert lens == want[0] and status == want[1]


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("P,H,D,layers,group_of,pad", FEW)
def test_many_rows(cache, P, H, D, layers, group_of, pad):
    """First and last tokens of long requests, every second one, all but one."""
    new, kv_len = [1500, 700, 431], [1500, 733, 440]
    kept = [[0, 1, 2, 3] + list(range(1200, 1500)), list(range(0, 700, 2)), [k for k in range(431) if k != 5]]
    c, tables = make(3, P, H, D, cache, new, kv_len, layers, group_of, pad)
    lens, status, want = run(c, tables, new, kv_len, kept)
    assert lens == want[0] and status == want[1] and set(status) == {T.ACCEPT}


@pytest.mark.parametrize("cache,H,D,new,layers", [("fp8_scaled", 4, 128, 90, 2), ("fp8_scaled", 2, 256, 90, 2), ("fp8_scaled", 6, 64, 90, 2), ("bf16", 4, 128, 90, 2),
                                                  ("fp8_scaled", 16, 128, 300, 17), ("bf16", 16, 64, 300, 33), ("fp8_scaled", 3, 64, 300, 1),
                                                  ("fp8_scaled", 3, 256, 300, 1), ("bf16", 3, 128, 300, 1)])
@pytest.mark.parametrize("P", [16, 104])
def test_both_sides_of_the_rules(cache, H, D, new, layers, P):
    """Requests of some and of many rows, few and many workgroups, pages of fewer and more rows than a step."""
    if cache == "bf16" and P * H * D % 512:
        pytest.skip("slabs are whole KiB")
    r = np.random.default_rng(15)
    news = [new, new + 17, new + 40, new]
    kv_len = [a + int(h) for a, h in zip(news, r.integers(0, 40, 4))]
    kept = [some(r, news[0], 40), list(range(news[1] // 2, news[1])), some(r, news[2], 9), [0, 1] + list(range(30, news[3], 2))]
    c, tables = make(16, P, H, D, cache, news, kv_len, layers=layers)
    lens, status, want = run(c, tables, news, kv_len, kept)
    assert lens == want[0] and status == want[1] and set(status) == {T.ACCEPT}


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("P", [16, 104])
@pytest.mark.parametrize("more", [1, 10])
def test_entries_that_cannot_be_kept(cache, P, more):
    """Tokens before the first of them are kept in all layers, whichever layers' table lacks the page."""
    new = [40 * more, 40 * more, 40 * more, 12 * more, 30 * more, 9, 20 * more, 5]
    kv_len = [a + 20 for a in new]
    kept = [[0, 5, 5, 9], [3, 2, 8], [0, 1, 2, 40 * more], list(range(2, 12)) + [2 ** 32 - 1], [1, 6, 20, 29 * more], [0, 4], [0, 3], [1, 4]]
    c, tables = make(4, P, 4, 64, cache, new, kv_len, 3, [0, 1, 0])
    tables[1, 4, (kv_len[4] - new[4] + 20) // P] = -1
    kv_len[5] = 8  # fewer than its new tokens
    kv_len[6] = tables.shape[2] * P + 5  # past its row
    lens, status, want = run(c, tables, new, kv_len, kept)
    assert lens == want[0] and status == want[1]
    assert status == [T.BADARG] * 7 + [T.ACCEPT]


def test_more_kept_than_there_are():
    new, kv_len = [4, 3], [20, 19]
    c, tables = make(5, 16, 4, 64, "fp8_scaled", new, kv_len)
    lens, status, want = run(c, tables, new, kv_len, [[0, 2, 3], [0, 1, 2]], n_keep=[3, 4])
    assert status == [T.ACCEPT, T.BADARG] and lens == want[0]


@pytest.mark.parametrize("P", [16, 104, 256])
def test_scales_of_every_size(P):
    """Scale bytes over their whole range and beside it, values that are NaN, heads of zeros."""
    new, kv_len = [300, 60], [310, 75]
    c, tables = make(6, P, 4, 64, "fp8_scaled", new, kv_len)
    s = slice(c.code_bytes, c.code_bytes + 4)
    c.host[:, :, s] = c.r.integers(0, 256, c.host[:, :, s].shape)
    codes = c.host[:, :, :c.code_bytes].reshape(4, c.n_pages, P, 4, 64)
    codes[:, :, :, 0] &= 0x80  # zeros
    codes[:, ::2, :, 1] &= 0x83  # below the smallest normal code
    codes[:, :, ::3, 2] |= 0x7F  # NaN
    c.up()
    r = np.random.default_rng(8)
    lens, status, want = run(c, tables, new, kv_len, [some(r, 300, 130), some(r, 60, 11)])
    assert lens == want[0] and status == want[1]


def test_no_requests_and_no_rows():
    c, tables = make(7, 16, 4, 64, "bf16", [2], [2])
    lens, status, want = run(c, np.repeat(tables, 2, 1), [0, 0], [0, 5], [[], []])
    assert lens == [0, 5] and status == [T.ACCEPT, T.ACCEPT]


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("long", [False, True])
def test_captured_on_a_stream_of_its_own(cache, long):
    """Replayed with other entries, lengths and tables; every replay against the host."""
    r = np.random.default_rng(11)
    new = [700, 40] if long else [12, 7]
    kv_len = [a + 21 for a in new]
    c, tables = make(12, 16, 4, 64, cache, new, kv_len)
    off = np.concatenate([[0], np.cumsum(new)])
    d_keep, d_n, d_len, d_tab = up(np.zeros(sum(new))), up(np.zeros(2)), up(np.array(kv_len)), up(tables)
    batch, pages = T.make_batch(2, sum(new), up(off), d_len, d_tab, tables.shape[2]), c.paged.tl()
    out, status = up(np.zeros(2)), torch.zeros(2, dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        T.tl_keep(c.ctx, side, batch, pages, d_n, d_keep, out, status)
    for turn in range(4):
        kept = [some(r, n, int(r.integers(1, n // 2))) for n in new]
        kv = [k - int(r.integers(0, 5)) for k in kv_len]
        flat = np.zeros(sum(new), np.int64)
        for i, k in enumerate(kept):
            flat[off[i]:off[i] + len(k)] = k
        # the other order of each request's pages behind its first
        for g in range(c.groups):
            for i in range(2):
                at = np.flatnonzero(tables[g, i] >= 0)
                tables[g, i, at[1:]] = tables[g, i, at[1:]][::-1]
        for x, y in ((d_keep, flat), (d_n, np.array([len(k) for k in kept])), (d_len, np.array(kv)), (d_tab, tables)):
            x.copy_(up(y))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = hc.keep(c, tables, new, kv, kept)
        assert out.tolist() == want[0] and status.tolist() == want[1], turn
        c.same("replay %d" % turn)


@pytest.mark.parametrize("long", [False, True])
def test_offsets_past_32_bits(long):
    """Pages beyond the first 4 GiB of a cache."""
    from paper_2609_39358_amd.device import PagedCache

    r = np.random.default_rng(13)
    new = [600] if long else [20]
    kept = [some(r, new[0], new[0] // 3)]
    c, tables = make(14, 16, 8, 128, "fp8_scaled", new, [new[0] + 9], layers=1)
    n_pages = (9 << 29) // c.stride
    big = [torch.empty((n_pages, c.stride), dtype=torch.uint8, device=DEV) for _ in range(2)]
    for b, x in zip(big, c.dev):
        b[n_pages - c.n_pages:] = x
    far = np.where(tables >= 0, tables + (n_pages - c.n_pages), -1)
    paged = PagedCache(1, n_pages, c.stride, DEV, [big[0]], [big[1]])
    lens = up(np.zeros(1))
    batch = T.make_batch(1, new[0], up(np.array([0, new[0]])), up(np.array([new[0] + 9])), up(far), far.shape[2])
    T.tl_keep(c.ctx, torch.cuda.current_stream(), batch, paged.tl(), up(np.array([len(kept[0])])), up(np.array(kept[0] + [0] * (new[0] - len(kept[0])))), lens)
    torch.cuda.synchronize()
    want = hc.keep(c, tables, new, [new[0] + 9], kept)
    c.dev = torch.stack([b[n_pages - c.n_pages:] for b in big])
    c.same()
    assert lens.tolist() == want[0]
