"""tl_attend with a tree against 64 bits: trees over caches of every head size and page
size, on every kernel; masks that are no trees, name nothing, or have no word for a
token; windows; missing pages; values that are not finite; equal to tl_attend where the
masks are a text's; captured and replayed."""
import math

import numpy as np
import pytest
import torch

from paper_2609_39358_amd import taliesin as T
from tests import paged_case as pc
from tests.paged_case import DEV, Paged

pytestmark = pytest.mark.gpu


def up(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def drafted(r, new, back=8):
    """[new][new] which new token a row sees (itself and its ancestors), and depths."""
    see, depth = np.zeros((new, new), bool), np.zeros(new, int)
    for i in range(new):
        see[i, i] = True
        if i:
            p = int(r.integers(max(0, i - back), i))
            see[i] |= see[p]
            depth[i] = depth[p] + 1
    return see, depth


def words_of(see, words):
    out = np.zeros((see.shape[0], words), np.uint64)
    for j in range(min(see.shape[1], 64 * words)):
        out[:, j // 64] |= see[:, j].astype(np.uint64) << np.uint64(j % 64)
    return out


def attend(c, q, scale, see, depth, words):
    """As paged_case.attend, with masks: (out, lse, bounds of their errors)."""
    rows, Hq, D = q.shape
    G = Hq // c.H
    out, lse = np.zeros((rows, Hq, D)), np.full((rows, Hq), -np.inf)
    tol, ltol = np.zeros((rows, Hq, D)), np.zeros((rows, Hq))
    at = 0
    for i in range(c.n):
        k, v = c.values(0, i), c.values(1, i)
        named = np.repeat((c.table[i] >= 0) & (c.table[i] < c.n_pages), c.P)[:c.kv_len[i]]
        before = c.kv_len[i] - c.q_len[i]
        j = np.arange(c.kv_len[i])
        for t in range(c.q_len[i]):
            seen = (j < before) & (j > before + depth[i][t] - c.window if c.window else True)
            new = np.zeros(c.q_len[i], bool)
            n = min(c.q_len[i], 64 * words)
            new[:n] = see[i][t, :n]
            seen[max(before, 0):] |= new[max(-before, 0):]
            seen &= named
            if not seen.any():
                continue
            for h in range(Hq):
                kk, vv = k[seen, h // G], v[seen, h // G]
                x = q[at + t, h]
                s = kk @ x * scale
                size = (np.abs(kk) @ np.abs(x)).max() * abs(scale)
                ds = size * 2.0 ** -19 + 2.0 ** -20 * (np.abs(s).max() + 16)
                w = np.exp(s - s.max())
                out[at + t, h] = w @ vv / w.sum()
                lse[at + t, h] = s.max() + math.log(w.sum())
                # weights and results are rounded to bf16, half a step of 2^-8 each; scores are off by ds
                tol[at + t, h] = (w @ np.abs(vv) / w.sum()) * (2 * 2.0 ** -8 * 1.01 + 2 * ds) + 1e-30
                ltol[at + t, h] = 2 * ds + 1e-5
        at += c.q_len[i]
    return out, lse, tol, ltol


def call(c, q, Hq, words, masks, depth, scale=None, stream=None, pos=None):
    D = c.D
    out = torch.full((c.rows, Hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((c.rows, Hq), 7.0, device=DEV)
    size = T.tl_attend_workspace_bytes(c.ctx, Hq, c.n, c.rows)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV)
    if pos is None:
        pos = np.concatenate([k - n + np.asarray(d) for n, k, d in zip(c.q_len, c.kv_len, depth)]).astype(np.int32)
    tree = T.make_tree(up(masks.view(np.int64)), up(pos) if c.window else None)
    T.tl_attend(c.ctx, stream, c.layer, c.batch(), c.paged.tl(), q, out, ws, size, scale=scale, lse=lse, tree=tree)
    torch.cuda.synchronize()
    return out, lse


def check(c, Hq, see, depth, words, scale=None, extra=None):
    x = torch.from_numpy((c.r.standard_normal((c.rows, Hq + 2, c.D)) * 1.5).astype(np.float32)).to(torch.bfloat16)
    q = x.to(DEV)[:, 1:1 + Hq]
    masks = np.concatenate([words_of(s, words) for s in see])
    if extra is not None:
        masks = extra(masks)
    out, lse = call(c, q, Hq, words, masks, depth, scale)
    host = x[:, 1:1 + Hq].float().numpy().astype(float)
    want, wlse, tol, ltol = attend(c, host, c.D ** -0.5 if scale is None else scale, see, depth, words)
    got, glse = out.float().cpu().numpy(), lse.cpu().numpy()
    none = np.isneginf(wlse)
    assert np.array_equal(np.isneginf(glse), none)
    assert (np.abs(glse[~none] - wlse[~none]) <= ltol[~none]).all()
    bad = np.argwhere(~(np.abs(got - want) <= tol))
    assert bad.size == 0, (len(bad), bad[:3], got[tuple(bad[0])], want[tuple(bad[0])])


def trees(c, r, back=8):
    both = [drafted(r, n, back) for n in c.q_len]
    return [b[0] for b in both], [b[1] for b in both]


SHAPES = [  # P, H, D, Hq, pad
    (16, 4, 64, 8, 0),
    (16, 8, 128, 32, 0),
    (16, 16, 128, 32, 0),
    (104, 1, 64, 8, 16),
    (32, 6, 256, 24, 1024),
    (256, 2, 128, 2, 0),
    (7, 8, 64, 16, 0),
    (1, 4, 128, 8, 0),
]
BATCHES = {  # new tokens, cached tokens before them
    "few": ([1, 2, 5, 8, 3], [0, 1, 63, 200, 31]),
    "one": ([8], [1025]),
    "wide": ([64, 1, 33, 0, 70], [100, 17, 0, 3, 333]),
    "large": ([129, 200, 65], [64, 700, 1]),
}


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("name", list(BATCHES))
@pytest.mark.parametrize("P,H,D,Hq,pad", SHAPES)
def test_trees(cache, name, P, H, D, Hq, pad):
    new, before = BATCHES[name]
    c = Paged(1, P, H, D, cache, new, [a + b for a, b in zip(new, before)], pad=pad, layers=2, layer=1, group_of=[0, 1]).fill(spread=2).up()
    see, depth = trees(c, np.random.default_rng(2))
    check(c, Hq, see, depth, -(-max(new) // 64))


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("name", list(BATCHES))
@pytest.mark.parametrize("P,H,D,Hq", [(16, 2, 128, 8), (104, 1, 64, 8), (32, 2, 256, 4)])
@pytest.mark.parametrize("window", [1, 40, 300])
def test_windows(cache, name, P, H, D, Hq, window):
    """From a row's own position, for the tokens before the tree; a window smaller than a depth
    leaves none of those, and the new tokens are the masks' matter."""
    new, before = BATCHES[name]
    c = Paged(3, P, H, D, cache, new, [a + b for a, b in zip(new, before)], window=window).fill(spread=1).up()
    see, depth = trees(c, np.random.default_rng(4), 3)
    check(c, Hq, see, depth, -(-max(new) // 64))


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("H,D,Hq,n,new", [(16, 64, 16, 40, 3), (16, 64, 32, 90, 5), (6, 128, 6, 60, 2), (16, 64, 16, 21, 70), (16, 128, 32, 10, 71), (16, 128, 32, 17, 66),
                                          (16, 256, 16, 10, 20), (1, 256, 4, 170, 6)])
def test_windows_of_many_requests(cache, ragged, H, D, Hq, n, new):
    """As many tiles as workgroups, or some times as many: on each kernel."""
    r = np.random.default_rng(17)
    news = [int(x) for x in r.integers(0, 2 * new, n)] if ragged else [new] * n
    c = Paged(18, 16, H, D, cache, news, [a + int(b) for a, b in zip(news, r.integers(0, 120, n))], window=50).fill(spread=1).up()
    see, depth = trees(c, r, 3)
    check(c, Hq, see, depth, -(-max(news) // 64))


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("name", list(BATCHES))
@pytest.mark.parametrize("P,H,D,Hq", [(16, 2, 128, 8), (104, 1, 64, 8), (32, 2, 256, 4)])
def test_any_masks(cache, name, P, H, D, Hq):
    """Random bits: rows that see later rows, not themselves, or nothing; bits past the request's
    rows mean nothing, and tokens past the masks' words are not seen."""
    new, before = BATCHES[name]
    c = Paged(5, P, H, D, cache, new, [a + b for a, b in zip(new, before)]).fill().up()
    r = np.random.default_rng(6)
    see = [r.random((n, n)) < 0.4 for n in new]
    for s in see:
        s[1::5] = False
    for words in (1, 4):
        def extra(m):
            at = 0
            for n in new:
                for j in range(n, 64 * words):
                    m[at:at + n, j // 64] |= np.uint64(1) << np.uint64(j % 64)
                at += n
            return m
        check(c, Hq, see, [np.zeros(n, int) for n in new], words, extra=extra)


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("D,Hq", [(64, 8), (128, 8), (256, 4)])
@pytest.mark.parametrize("many", [False, True])
def test_missing_pages_and_nothing_before(cache, D, Hq, many):
    new = [70, 100, 64] if many else [4, 9, 1]
    kv_len = [new[0] + 40, new[1], new[2] + 33]
    c = Paged(7, 16, 2, D, cache, new, kv_len).fill()
    c.table[0, 1], c.table[0, (40 + new[0] // 2) // 16], c.table[2, :3] = -1, c.n_pages, -1
    c.up()
    see, depth = trees(c, np.random.default_rng(8))
    see[1][3:] = False  # rows that see nothing at all
    check(c, Hq, see, depth, 2)
    check(c, Hq, see, depth, 2, scale=-0.3)


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("D,Hq", [(64, 8), (128, 8), (256, 4)])
@pytest.mark.parametrize("new", [1, 6, 90])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(cache, D, Hq, new):
    """Keys and values of drafted tokens that are NaN (or infinite): rows that do not see the token
    are as if it were not there; those that do are NaN (infinite) there."""
    P, H, before = 16, 2, 45
    c = Paged(9, P, H, D, cache, [new], [before + new]).fill()
    r = np.random.default_rng(10)
    see, depth = drafted(r, new, 4)
    bad_v, bad_k = new // 2, new - 1
    if new == 1:
        see[:] = False  # one row that sees neither itself
    x = torch.from_numpy(r.standard_normal((new, Hq, D)).astype(np.float32)).to(torch.bfloat16).to(DEV)
    c.up()
    masks = words_of(see, 2)
    want, wlse = call(c, x, Hq, 2, masks, [depth])
    code = 0x7FC0 if cache == "bf16" else 0x7F
    at = before + bad_v
    c.codes(1)[c.table[0, at // P], at % P, 1, 3] = code
    if cache == "bf16":
        c.codes(1)[c.table[0, at // P], at % P, 0, 5] = 0x7F80
    at = before + bad_k
    c.codes(0)[c.table[0, at // P], at % P, 0, 7] = code
    c.up()
    got, glse = call(c, x, Hq, 2, masks, [depth])
    got, glse, want, wlse = (y.float().cpu().numpy() for y in (got, glse, want, wlse))
    G = Hq // H
    for t in range(new):
        sees_v, sees_k = see[t, bad_v], see[t, bad_k]
        nan = np.zeros((Hq, D), bool)
        if sees_v:
            nan[G:, 3] = True
        if sees_k:
            nan[:G] = True
        inf = np.zeros((Hq, D), bool)
        if sees_v and cache == "bf16":
            inf[:G, 5] = ~nan[:G, 5]
        assert np.array_equal(np.isnan(got[t]), nan), t
        assert (got[t][inf] == np.inf).all()
        rest = ~nan & ~inf
        assert np.array_equal(got[t][rest], want[t][rest]), t
        assert np.array_equal(np.isnan(glse[t]), np.repeat([sees_k, False], G))


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("D,H,Hq", [(64, 4, 8), (128, 8, 32), (256, 2, 8)])
@pytest.mark.parametrize("new", [[1, 1, 1], [3, 7, 1], [64, 90, 20], [300, 5, 128]])
@pytest.mark.parametrize("window", [0, 200])
def test_a_text_is_a_tree(cache, D, H, Hq, new, window):
    """Masks of all rows up to a row's own give tl_attend's results, within what either may be off."""
    c = Paged(11, 16, H, D, cache, new, [a + b for a, b in zip(new, [500, 0, 77])], window=window).fill().up()
    see, depth = [np.tril(np.ones((n, n), bool)) for n in new], [np.arange(n) for n in new]
    if window:
        see = [s & ~np.tril(s, -window) for s in see]
    x = torch.from_numpy(c.r.standard_normal((c.rows, Hq, D)).astype(np.float32)).to(torch.bfloat16)
    words = -(-max(new) // 64)
    out, lse = call(c, x.to(DEV), Hq, words, np.concatenate([words_of(s, words) for s in see]), depth)
    plain, plse = torch.empty_like(out), torch.empty_like(lse)
    size = T.tl_attend_workspace_bytes(c.ctx, Hq, c.n, c.rows)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    T.tl_attend(c.ctx, None, 0, c.batch(), c.paged.tl(), x.to(DEV), plain, ws, size, lse=plse)
    torch.cuda.synchronize()
    want, wlse, tol, ltol = attend(c, x.float().numpy().astype(float), D ** -0.5, see, depth, words)
    for o, l in ((out, lse), (plain, plse)):
        assert (np.abs(o.float().cpu().numpy() - want) <= tol).all() and (np.abs(l.cpu().numpy() - wlse) <= ltol).all()


def test_positions_outside_are_brought_inside():
    """Positions before or behind the new tokens' places are taken as the nearest of those."""
    new, before = [20], [100]
    c = Paged(13, 16, 2, 64, "bf16", new, [120], window=30).fill().up()
    see, _ = trees(c, np.random.default_rng(1))
    x = torch.from_numpy(c.r.standard_normal((20, 4, 64)).astype(np.float32)).to(torch.bfloat16).to(DEV)
    masks = words_of(see[0], 1)
    pos = np.array([-5, 2 ** 31 - 1, 99, 120, -2 ** 31] * 4, np.int32)
    a, _ = call(c, x, 4, 1, masks, None, pos=pos)
    b, _ = call(c, x, 4, 1, masks, None, pos=np.clip(pos, 100, 119))
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("new", [[7, 1, 3], [64, 33, 50]])
def test_captured(new):
    """Replayed with other lengths, tables and masks, eager calls between; rows that no request
    owns are left alone; on a stream of its own, with a workspace of its own."""
    c = Paged(15, 16, 2, 128, "fp8_scaled", new, [a + 200 for a in new]).fill().up()
    rows = c.rows + 5
    x = torch.from_numpy(c.r.standard_normal((rows, 8, 128)).astype(np.float32)).to(torch.bfloat16).to(DEV)
    r = np.random.default_rng(3)
    d_mask = torch.zeros((rows, 1), dtype=torch.int64, device=DEV)
    batch = T.make_batch(c.n, rows, *c.d, c.width)
    tree, cache = T.make_tree(d_mask), c.paged.tl()
    size = T.tl_attend_workspace_bytes(c.ctx, 8, c.n, rows)

    def buffers():
        return (torch.full((rows, 8, 128), 3.0, dtype=torch.bfloat16, device=DEV), torch.full((rows, 8), 3.0, device=DEV),
                torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV))

    (out, lse, ws), (out2, lse2, ws2) = buffers(), buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    T.tl_attend(c.ctx, side, 0, batch, cache, x, out, ws, size, lse=lse, tree=tree)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        T.tl_attend(c.ctx, torch.cuda.current_stream(), 0, batch, cache, x, out, ws, size, lse=lse, tree=tree)
    for i in range(4):
        see = [drafted(r, n)[0] for n in new]
        d_mask[:c.rows].copy_(up(np.concatenate([words_of(s, 1) for s in see]).view(np.int64)))
        c.d[1].copy_(up(np.array([a + int(r.integers(0, 200)) for a in new], np.int32)))
        T.tl_attend(c.ctx, torch.cuda.current_stream(), 0, batch, cache, x, out2, ws2, size, lse=lse2, tree=tree)
        out.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), out2.view(torch.int16)) and torch.equal(lse, lse2)
        assert (out[c.rows:] == 3.0).all() and torch.isfinite(out.float()).all()
