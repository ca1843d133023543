"""Values that are not finite at the ends of what a tile sees: blocks that are not
whole hold copies of a neighbouring key, which must not count."""
import numpy as np
import pytest
import torch

from paper_2609_39358_amd import taliesin as T
from tests import paged_case as pc
from tests.paged_case import DEV, Paged
from tests.test_gpu_attend import queries
from tests.test_gpu_attend_nan import compare

pytestmark = pytest.mark.gpu


def spoil(c, cache, i, keys):
    """Infinite (8 bits: NaN) values at some keys of request i, an element each."""
    for m, key in enumerate(keys):
        bits = [0x7F80, 0xFF80][m % 2] if cache == "bf16" else 0x7F
        c.codes(1)[c.table[i, key // c.P], key % c.P, m % c.H, (5 * m + 2) % c.D] = bits


ALL = [  # P, H, D, Hq, q_len, kv_len
    (16, 2, 64, 4, [40, 50, 33], [70, 129, 40]),    # four wavefronts
    (16, 2, 128, 4, [100, 3, 90], [17, 200, 130]),  # eight
    (104, 1, 128, 4, [150, 1], [209, 105]),
    (32, 3, 256, 6, [20, 33, 1], [75, 1, 31]),
    (16, 2, 64, 4, [1, 1, 5], [130, 7, 40]),        # tiles of 16 rows
]


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("P,H,D,Hq,q_len,kv_len", ALL)
def test_all_keys(cache, P, H, D, Hq, q_len, kv_len):
    c = Paged(50, P, H, D, cache, q_len, kv_len).fill()
    for i, k in enumerate(kv_len):
        spoil(c, cache, i, [k - 1] if i != 1 else [k - 1, 0, k // 2])
    c.up()
    d, q = queries(c, Hq)
    want = compare(c, d, q, all_keys=True)
    assert not np.isfinite(want).all() and np.isfinite(want).any()


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("window", [0, 30])
def test_tiles_of_one_token(cache, window):
    """More query heads than a tile has rows: a tile is one token, whose own key is its last."""
    c = Paged(51, 16, 1, 64, cache, [1, 40], [40, 90], window).fill()
    spoil(c, cache, 0, [39, 12])
    spoil(c, cache, 1, [89, 60, 71])
    c.up()
    d, q = queries(c, 130)
    want = compare(c, d, q)
    assert not np.isfinite(want).all() and np.isfinite(want).any()


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("H,D,rows", [(2, 64, 60), (2, 128, 150), (1, 256, 60)])
def test_lengths_past_the_end_of_a_table_row(cache, H, D, rows):
    """Lengths are cut to what a table row names: rows behind its end see all of it."""
    held, Hq = 80, 4 * H
    c = Paged(52, 16, H, D, cache, [rows], [held]).fill()
    spoil(c, cache, 0, [held - 1, 3])
    c.up()
    d, q = queries(c, Hq)
    out = torch.empty((rows, Hq, D), dtype=torch.bfloat16, device=DEV)
    n = T.tl_attend_workspace_bytes(c.ctx, Hq, 1, rows)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)
    c.d[1].fill_(held + rows + 33)
    T.tl_attend(c.ctx, None, 0, c.batch(), c.paged.tl(), d, out, ws, n)
    got = out.float().cpu().numpy()
    with np.errstate(invalid="ignore"):
        want, _, tol, _ = pc.attend(c, q, D ** -0.5, all_keys=True)
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
        assert (np.abs(got - want) <= tol)[np.isfinite(want)].all()
