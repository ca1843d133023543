"""tl_attend against attention in 64 bits on the host, within bounds that follow
from what the kernels round, over head sizes, caches, page sizes, ragged batches,
windows, missing pages, empty rows, and lengths that one workgroup or many share."""
import numpy as np
import pytest
import torch

from paper_2609_39358_amd import taliesin as T
from paper_2609_39358_amd.device import PagedCache
from tests import paged_case as pc
from tests.paged_case import DEV, Paged

pytestmark = pytest.mark.gpu


def run(c, q, scale=None, all_keys=False, lse=True, ws_fill=0xFF, rows=None, cache=None, stream=None):
    """(out, lse) of one call; the workspace holds NaN before it."""
    n, Hq, D = q.shape
    out = torch.full((n, Hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    d_lse = torch.full((n, Hq), 7.0, device=DEV) if lse else None
    ws_b = T.tl_attend_workspace_bytes(c.ctx, Hq, c.n, n)
    ws = torch.full((ws_b,), ws_fill, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    T.tl_attend(c.ctx, stream, c.layer, c.batch(n), cache or c.paged.tl(), q, out, ws, ws_b, scale, d_lse, all_keys)
    torch.cuda.synchronize()
    return out.float().cpu().numpy(), None if d_lse is None else d_lse.cpu().numpy()


def queries(c, Hq, amp=1.5):
    q = torch.from_numpy((c.r.standard_normal((c.rows, Hq, c.D)) * amp).astype(np.float32)).to(torch.bfloat16)
    return q.to(DEV), q.float().numpy().astype(float)


def check(c, Hq, all_keys=False, scale=None, amp=1.5):
    d, q = queries(c, Hq, amp)
    print("attend", c.cache, c.P, c.H, c.D, Hq, c.q_len[:4], c.kv_len[:4], c.window, all_keys, flush=True)
    got, lse = run(c, d, scale, all_keys)
    want, wlse, tol, ltol = pc.attend(c, q, c.D ** -0.5 if scale is None else scale, all_keys)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4], got[bad][:4], want[bad][:4])
    empty = np.isneginf(wlse)
    assert np.array_equal(empty, np.isneginf(lse))
    bad = ~empty & ~(np.abs(np.where(empty, 0, lse) - np.where(empty, 0, wlse)) <= ltol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4], lse[bad][:4], wlse[bad][:4])
    return got


SHAPES = [  # P, H, D, Hq, q_len, kv_len, window, pad
    (16, 4, 64, 8, [1], [1], 0, 0),
    (16, 4, 64, 8, [1, 1, 1, 0, 1], [1, 127, 128, 9, 700], 0, 0),
    (16, 2, 128, 8, [1] * 9, [3, 1, 600, 31, 32, 33, 129, 256, 257], 0, 0),
    (16, 2, 128, 8, [3, 1, 2], [3, 64, 200], 0, 0),
    (16, 2, 128, 4, [70, 1, 130], [70, 300, 391], 0, 0),
    (104, 1, 64, 8, [1, 2], [105, 320], 0, 0),
    (104, 2, 64, 12, [40, 99], [250, 99], 0, 0),
    (32, 3, 256, 12, [1, 1], [95, 33], 0, 1024),
    (32, 2, 256, 6, [45, 64], [77, 64], 0, 1024),
    (256, 2, 128, 4, [1, 1], [300, 900], 130, 0),
    (256, 2, 128, 4, [100, 33], [400, 33], 64, 0),
    (16, 1, 64, 20, [1, 3], [50, 200], 1, 0),
    (7, 8, 64, 8, [30], [45], 10, 16),
    (16, 1, 64, 130, [1, 2], [40, 35], 0, 0),
    (16, 1, 64, 130, [1, 40], [40, 90], 0, 0),
    (1, 8, 64, 8, [1, 17], [20, 17], 0, 0),
]


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("P,H,D,Hq,q_len,kv_len,window,pad", SHAPES)
def test_attend(cache, P, H, D, Hq, q_len, kv_len, window, pad):
    c = Paged(2, P, H, D, cache, q_len, kv_len, window, pad=pad, layers=2, layer=1, group_of=[1, 0]).fill(spread=1).up()
    check(c, Hq)


SIDES = [  # P, H, D, Hq, q_len, kv_len: both sides of the sizes where other tiles or numbers of workgroups are taken
    (16, 2, 64, 4, [32, 32], [300, 200]),
    (16, 2, 64, 4, [33, 33], [300, 200]),
    (16, 1, 64, 2, [2048], [2100]),
    (16, 1, 64, 2, [2049], [2100]),
    (16, 1, 128, 4, [8, 8], [1500, 60]),
    (16, 1, 128, 4, [9, 9], [1500, 60]),
    (16, 1, 128, 4, [33], [400]),
    (32, 1, 256, 4, [3, 3], [900, 33]),
    (32, 1, 256, 4, [4, 4], [900, 33]),
    (16, 8, 64, 16, [1], [2000]),
    (16, 8, 64, 64, [2], [2000]),
    (16, 8, 128, 64, [2], [2000]),
    (16, 8, 128, 64, [2] * 40, [100 + i for i in range(40)]),
]


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("P,H,D,Hq,q_len,kv_len", SIDES)
def test_both_sides_of_the_rules(cache, P, H, D, Hq, q_len, kv_len):
    check(Paged(28, P, H, D, cache, q_len, kv_len).fill(spread=1).up(), Hq)


CROSS = [
    (16, 2, 64, 4, [1, 1, 5], [130, 0, 40], 0),
    (32, 3, 256, 6, [20, 33, 1], [75, 0, 31], 0),
    (104, 1, 64, 8, [1] * 5, [104, 105, 3, 208, 1], 50),  # a window does not apply
    (16, 2, 128, 2, [90, 3], [17, 200], 0),
]


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("P,H,D,Hq,q_len,kv_len,window", CROSS)
def test_all_keys(cache, P, H, D, Hq, q_len, kv_len, window):
    c = Paged(4, P, H, D, cache, q_len, kv_len, window).fill().up()
    got = check(c, Hq, all_keys=True)
    at = 0
    for n, k in zip(q_len, kv_len):
        assert k or not got[at:at + n].any()
        at += n


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("q_len,Hq,H,D", [([1], 8, 2, 128), ([2, 1], 4, 2, 64), ([150], 4, 2, 128), ([40], 6, 1, 256)])
def test_long_caches_are_shared_by_many_workgroups(cache, q_len, Hq, H, D):
    c = Paged(6, 16, H, D, cache, q_len, [9000 + 17 * i for i in range(len(q_len))]).fill().up()
    check(c, Hq)


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("q_len", [1, 60])
def test_many_requests(cache, q_len):
    """More requests than a workgroup has threads, of all lengths, some with no rows."""
    r = np.random.default_rng(8)
    kv = [int(k) for k in r.integers(q_len, 150, 600)]
    rows = [q_len if i % 7 == 1 else 0 for i in range(600)] if q_len > 1 else [int(i % 5 > 0) for i in range(600)]
    c = Paged(8, 16, 2, 64, cache, rows, kv).fill().up()
    check(c, 4)


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("q_len", [1, 50])
def test_missing_pages_are_left_out(cache, q_len):
    c = Paged(10, 16, 2, 128, cache, [q_len, q_len], [300, 200]).fill()
    c.table[0, [0, 3, 4, 9]] = [-1, -1, c.n_pages, 2 ** 31 - 1]
    c.table[1, :] = -1  # nothing restored: zeros
    c.up()
    got = check(c, 8)
    assert not got[q_len:].any()


@pytest.mark.parametrize("q_len", [[7], [40]])
def test_more_rows_than_keys(q_len):
    """Rows whose position is negative see nothing."""
    c = Paged(12, 16, 2, 64, "bf16", q_len, [5]).fill().up()
    got = check(c, 4)
    assert not got[:q_len[0] - 5].any()


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("q_len", [1, 64])
def test_large_scores(cache, q_len):
    """Scores of hundreds, rising along the cache and falling: the running maximum follows them."""
    for back in (False, True):
        c = Paged(14, 16, 1, 64, cache, [q_len], [400]).fill()
        for j in range(25):
            p = c.table[0, j]
            k = 24 - j if back else j
            x = c.r.standard_normal((16, 1, 64)).astype(np.float32) * (0.2 + 0.4 * k)
            if cache == "bf16":
                c.codes(0)[p] = pc.bf16_bits(x)
            else:
                c.codes(0)[p] = pc.e4m3_codes(x * 8)
                c.scales(0)[p] = 124
        c.up()
        check(c, 2, amp=4.0)


def test_scales_at_their_ends():
    """Values of 2^-117 and of 2^120 times a code."""
    c = Paged(16, 16, 2, 64, "fp8_scaled", [1, 40], [30, 100]).fill()
    for kv, h0, h1 in ((0, 127, 127), (1, 10, 240)):
        c.scales(kv)[:, 0], c.scales(kv)[:, 1] = h0 - 4 * (kv == 0), h1 - 4 * (kv == 0)
    c.up()
    check(c, 2)


ODD = [  # H, D, Hq, q_len, kv_len, window
    (2, 64, 4, [5, 1], [60, 33], 0),
    (2, 64, 8, [3, 2], [3, 200], 40),
    (1, 64, 20, [2], [50], 0),
    (2, 128, 8, [4], [4000], 0),
    (2, 128, 8, [45, 3], [45, 100], 0),
    (2, 128, 4, [300], [500], 0),
    (2, 128, 4, [150, 2], [400, 90], 64),
    (2, 128, 4, [150], [9000], 0),
    (2, 256, 6, [3], [70], 0),
    (1, 256, 6, [90], [130], 30),
]


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("H,D,Hq,q_len,kv_len,window", ODD)
def test_values_that_are_not_finite_reach_the_rows_that_see_them(cache, H, D, Hq, q_len, kv_len, window):
    """NaN and infinite values, and NaN keys, among the new tokens and before them:
    the rows that see them have them in the same elements, no other row has."""
    c = Paged(26, 16, H, D, cache, q_len, kv_len, window).fill()
    odd = [0x7FC0, 0x7F80, 0xFF80] if cache == "bf16" else [0x7F, 0xFF, 0x7F]
    for i, (n, k) in enumerate(zip(q_len, kv_len)):
        first = k - n
        # a value before the new tokens only leaves the rows of a window
        for m, at in enumerate([k - 1, k - 1, first + n // 2] + ([first - 3, first - window + n // 3] if window and first > window else [])):
            c.codes(1)[c.table[i, at // 16], at % 16, m % H, 7 * m + 3] = odd[m % 3]
        at = first + 2 * n // 3
        if n > 1 and i == 0:
            c.codes(0)[c.table[i, at // 16], at % 16, 0, 5] = odd[0]
    c.up()
    d, q = queries(c, Hq)
    got, lse = run(c, d)
    with np.errstate(invalid="ignore"):
        want, wlse, tol, ltol = pc.attend(c, q, D ** -0.5)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        fine = np.isfinite(want)
        assert not fine.all() and fine.any()
        assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
        assert (np.abs(got - want) <= tol)[fine].all()
        assert np.array_equal(np.isnan(lse), np.isnan(wlse))
        assert (np.abs(lse - wlse) <= ltol)[np.isfinite(wlse)].all()


def test_strides_and_rows_of_no_request():
    c = Paged(18, 16, 2, 64, "bf16", [3, 50], [20, 90]).fill().up()
    Hq, n = 4, c.rows + 5
    wide = torch.randn((n, Hq + 4, 64), device=DEV).to(torch.bfloat16)
    q = wide[:, 2:2 + Hq]
    heads_first = torch.full((Hq, n, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    out = heads_first.transpose(0, 1)
    ws_b = T.tl_attend_workspace_bytes(c.ctx, Hq, c.n, n)
    ws = torch.full((ws_b,), 0xFF, dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    T.tl_attend(c.ctx, side, 0, c.batch(n), c.paged.tl(), q, out, ws, ws_b)
    side.synchronize()
    got = out.float().cpu().numpy()
    want, _, tol, _ = pc.attend(c, q[:c.rows].float().cpu().numpy().astype(float), 0.125)
    assert (np.abs(got[:c.rows] - want) <= tol).all()
    assert (got[c.rows:] == 7.0).all()


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("q_len", [1, 60])
def test_offsets_past_32_bits(cache, q_len):
    P, H, D = 16, 8, 128
    c = Paged(20, P, H, D, cache, [q_len], [200]).fill()
    n_pages = (9 << 29) // c.stride
    big = [torch.empty((n_pages, c.stride), dtype=torch.uint8, device=DEV) for _ in range(2)]
    small = c.table.copy()
    c.table = np.where(small >= 0, n_pages - 1 - small, -1).astype(np.int32)
    c.up()
    for b, p in zip(big, c.pages):
        b[n_pages - c.n_pages:] = torch.from_numpy(p[::-1].copy()).to(DEV)
    paged = PagedCache(1, n_pages, c.stride, DEV, [big[0]], [big[1]])
    d, q = queries(c, 8)
    got, _ = run(c, d, cache=paged.tl())
    c.table = small
    want, _, tol, _ = pc.attend(c, q, D ** -0.5)
    assert (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("q_len", [1, 60])
def test_same_bytes_every_time(q_len):
    c = Paged(22, 16, 4, 128, "fp8_scaled", [q_len] * 3, [3000, 100, 777]).fill().up()
    d, _ = queries(c, 8)
    a, la = run(c, d)
    for fill in (0, 0x7F):
        b, lb = run(c, d, ws_fill=fill)
        assert np.array_equal(a, b) and np.array_equal(la, lb)


@pytest.mark.parametrize("q_len", [1, 60])
def test_graph_replays_with_other_contents(q_len):
    """A captured append and attention, replayed with other lengths, tables and rows."""
    P, H, D, Hq = 16, 2, 64, 4
    c = Paged(24, P, H, D, "fp8_scaled", [q_len, q_len], [300, 170]).fill().up()
    n = c.rows
    x = torch.zeros((n, Hq + 2 * H, D), dtype=torch.bfloat16, device=DEV)
    q = torch.empty((n, Hq, D), dtype=torch.bfloat16, device=DEV)
    out = torch.empty_like(q)
    ws_b = T.tl_attend_workspace_bytes(c.ctx, Hq, c.n, n)
    ws = torch.empty(ws_b, dtype=torch.uint8, device=DEV)
    batch, cache = c.batch(), c.paged.tl()

    def step(out, q):
        s = torch.cuda.current_stream()
        T.tl_append(c.ctx, s, 0, batch, cache, x[:, Hq:Hq + H], x[:, Hq + H:], None, x[:, :Hq], q)
        T.tl_attend(c.ctx, s, 0, batch, cache, q, out, ws, ws_b)

    step(out, q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, q)
    for i, lens in enumerate(([300, 170], [280, 61], [299, 100], [300, 170])):
        c.d[1].copy_(torch.tensor(lens, dtype=torch.int32))
        x.copy_(torch.randn(x.shape, device=DEV) * (1 + i))
        k0, v0 = c.dk.clone(), c.dv.clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got, gk = out.clone(), c.dk.clone()
        c.dk.copy_(k0)
        c.dv.copy_(v0)
        eager, eq = torch.empty_like(out), torch.empty_like(q)
        step(eager, eq)
        torch.cuda.synchronize()
        assert torch.equal(got, eager) and torch.equal(gk, c.dk), i
