"""Trees and kept rows behind the longest requests, and lengths past those."""
import numpy as np
import pytest
import torch

from paper_2609_39358_amd import taliesin as T
from tests.paged_case import DEV
from tests.test_gpu_longest_requests import D, MOST, WINDOW, make
from tests.test_gpu_tree import drafted, words_of

pytestmark = pytest.mark.gpu


def words(x):
    return torch.tensor(x, dtype=torch.int64).to(torch.int32).to(DEV)


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("P", [65536, 65528])
@pytest.mark.parametrize("n", [1, 3, 20, 60, 200])
def test_trees(cache, P, n):
    ctx, paged, table, width, (k, v), first, r = make(P, cache)
    Hq = 2
    x = torch.from_numpy(r.standard_normal((n, Hq, D)).astype(np.float32) * 1.5).to(torch.bfloat16)
    d, q = x.to(DEV), x.double().numpy()
    see, depth = drafted(r, n)
    masks = torch.from_numpy(words_of(see, 4).view(np.int64)).to(DEV)
    for length in (MOST, MOST - 7):
        before = length - n
        tree = T.make_tree(masks, words([before + int(t) for t in depth]))
        batch = T.make_batch(1, n, words([0, n]), words([length]), table, width)
        ws_b = T.tl_attend_workspace_bytes(ctx, Hq, 1, n)
        ws, out = torch.empty(ws_b, dtype=torch.uint8, device=DEV), torch.empty_like(d)
        T.tl_attend(ctx, None, 0, batch, paged.tl(), d, out, ws, ws_b, tree=tree)
        got = out.double().cpu().numpy()
        for t in range(n):
            seen = np.zeros(len(k), bool)
            seen[max(0, before + depth[t] - WINDOW + 1 - first):before - first] = True
            seen[before - first:length - first] = see[t]
            s = k[seen] @ q[t].T * D ** -0.5  # [keys, heads]
            w = np.exp(s - s.max(0))
            want, size = (w.T @ v[seen]) / w.sum(0)[:, None], (w.T @ np.abs(v[seen])) / w.sum(0)[:, None]
            # weights and result rounded to bf16, half a step of 2^-8 each; 32-bit sums
            assert (np.abs(got[t] - want) <= size * (2 * 2.0 ** -8 * 1.01 + 2.0 ** -12) + 1e-30).all(), (length, t)


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("n", [3, 60])
def test_lengths_past_the_longest(cache, n):
    ctx, paged, table, width, _, _, r = make(65536, cache)
    table[:] = table[0, 0, (MOST - 1) // 65536]  # all tokens have a page
    for x in paged.k + paged.v:
        x.zero_()
    q = torch.from_numpy(r.standard_normal((n, 2, D)).astype(np.float32)).to(torch.bfloat16).to(DEV)
    masks = torch.full((n, 1), -1, dtype=torch.int64, device=DEV)
    ws_b = T.tl_attend_workspace_bytes(ctx, 2, 1, n)
    ws, out = torch.empty(ws_b, dtype=torch.uint8, device=DEV), torch.full((n, 2, D), 7.0, dtype=torch.bfloat16, device=DEV)
    for length in (MOST + 5, 2 ** 31 - 1, -1):  # -1: 2^32 - 1
        batch = T.make_batch(1, n, words([0, n]), words([length]), table, width)
        T.tl_attend(ctx, None, 0, batch, paged.tl(), q, out, ws, ws_b, tree=T.make_tree(masks, words([2 ** 31 - 1] * n)))
        lens, status = words([3]), torch.zeros(1, dtype=torch.uint8, device=DEV)
        T.tl_keep(ctx, None, batch, paged.tl(), words([2]), words([0, 2] + [0] * (n - 2)), lens, status)
        torch.cuda.synchronize()
        assert bool((out == 0).all())  # values of 0, or none
        assert status.tolist() == [T.BADARG] and lens.tolist() == [length]


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
def test_kept_rows(cache):
    ctx, paged, table, width, _, first, _ = make(65536, cache)
    n, before = 40, [x.clone() for x in paged.k + paged.v]
    kept = [0, 1, 7, 20, 39]
    batch = T.make_batch(1, n, words([0, n]), words([MOST]), table, width)
    lens, status = words([0]), torch.zeros(1, dtype=torch.uint8, device=DEV)
    T.tl_keep(ctx, None, batch, paged.tl(), words([5]), words(kept + [0] * 35), lens, status)
    torch.cuda.synchronize()
    assert status.tolist() == [T.ACCEPT] and lens.tolist() == [MOST - n + 5]
    row = D * (2 if cache == "bf16" else 1)
    at = 65536 - n  # of the last page, page 0
    for x, y in zip(paged.k + paged.v, before):
        for i, k in enumerate(kept):  # one page, one scale: codes move as they are
            y[0, (at + i) * row:(at + i + 1) * row] = y[0, (at + k) * row:(at + k + 1) * row].clone()
        assert torch.equal(x, y)
