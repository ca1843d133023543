"""Scores that are NaN reach the rows that see them whichever way a row's keys are
cut: one workgroup's, several workgroups' with a part that holds nothing but NaN,
several wavefronts'."""
import numpy as np
import pytest
import torch

from tests import paged_case as pc
from tests.paged_case import Paged
from tests.test_gpu_attend import queries, run

pytestmark = pytest.mark.gpu


def compare(c, d, q, all_keys=False):
    """Against the definition: NaN and infinities in the same places, the rest within its bounds."""
    got, lse = run(c, d, None, all_keys)
    with np.errstate(invalid="ignore"):
        want, wlse, tol, ltol = pc.attend(c, q, c.D ** -0.5, all_keys)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
        fine = np.isfinite(want)
        assert (np.abs(got - want) <= tol)[fine].all()
        assert np.array_equal(np.isnan(lse), np.isnan(wlse))
        assert np.array_equal(np.isneginf(lse), np.isneginf(wlse))
        assert (np.abs(lse - wlse) <= ltol)[np.isfinite(wlse)].all()
    return want


SHAPES = [  # H, D, Hq, q_len, kv_len, window
    (4, 64, 8, [1], [1024], 0),     # a decode row on 32 workgroups
    (1, 64, 8, [1], [40], 0),       # on one, its wavefronts share the head
    (1, 64, 8, [2, 1], [600, 9], 0),
    (3, 64, 6, [1], [700], 0),
    (2, 128, 8, [1, 1], [9000, 50], 0),
    (2, 128, 8, [3], [500], 130),
    (2, 64, 4, [150], [3000], 0),   # tiles of many rows, four wavefronts
    (2, 128, 4, [150], [9000], 0),  # eight
    (1, 256, 6, [1], [900], 0),
    (1, 256, 6, [90], [4000], 0),
]


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("H,D,Hq,q_len,kv_len,window", SHAPES)
def test_a_query_that_is_nan(cache, H, D, Hq, q_len, kv_len, window):
    c = Paged(40, 16, H, D, cache, q_len, kv_len, window).fill().up()
    d, q = queries(c, Hq)
    for t, h, e in ((0, 0, 3), (c.rows - 1, Hq - 1, D - 1), (c.rows // 2, 1, 0)):
        d[t, h, e] = float("nan")
        q[t, h, e] = np.nan
    want = compare(c, d, q)
    assert np.isnan(want).any() and np.isfinite(want).any()


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("H,D,Hq,q_len,kv_len,window", SHAPES)
def test_runs_of_keys_that_are_nan(cache, H, D, Hq, q_len, kv_len, window):
    """All keys of whole blocks, of one head, NaN: what a worker sees of a row may be nothing else."""
    c = Paged(41, 16, H, D, cache, q_len, kv_len, window).fill()
    first, n = max(0, kv_len[0] - q_len[0] - window) // 2 // 64 * 64, min(512, kv_len[0] // 3)
    if window:
        first, n = kv_len[0] - q_len[0] - window + 1, 1  # in the first row's window only
    for key in range(first, first + n):
        c.codes(0)[c.table[0, key // 16], key % 16, H - 1, key % D] = 0x7FC0 if cache == "bf16" else 0x7F
    c.up()
    d, q = queries(c, Hq)
    want = compare(c, d, q)
    assert np.isnan(want).any() and (H == 1 and not window and len(q_len) == 1 or np.isfinite(want).any())


def test_nothing_but_nan():
    """Every score of a row NaN, on one workgroup and on many."""
    for kv in (5, 64, 3000):
        c = Paged(42, 16, 2, 64, "bf16", [1], [kv]).fill().up()
        d, q = queries(c, 4)
        d.fill_(float("nan"))
        got, lse = run(c, d)
        assert np.isnan(got).all() and np.isnan(lse).all(), kv
    assert torch.isnan(d).all()
