"""tl_attend where its other tests have one head size only: pages that are not whole
sixteens of tokens, missing pages, and scales other than the usual one, in tiles of
16 rows and in tiles of many on four and on eight wavefronts."""
import pytest

from tests.paged_case import Paged
from tests.test_gpu_attend import check

pytestmark = pytest.mark.gpu

ODD_PAGES = [  # P, H, D, Hq, q_len, kv_len
    (104, 1, 128, 4, [1, 1, 2], [105, 1, 320]),
    (104, 1, 128, 8, [1], [5000]),  # shared by many workgroups
    (7, 4, 128, 16, [1] * 5, [1, 6, 7, 8, 500]),
    (104, 4, 128, 8, [1, 1], [209, 104]),
    (104, 1, 256, 6, [1, 1], [105, 700]),
    (7, 2, 256, 4, [1, 2], [300, 13]),
    (7, 4, 256, 8, [1], [4000]),
    (104, 1, 128, 4, [1, 90, 2], [208, 300, 105]),  # tiles of both kinds, four wavefronts
    (104, 1, 128, 4, [1, 300], [1000, 333]),        # eight
    (7, 4, 128, 8, [2, 1, 200], [9, 777, 200]),
    (104, 1, 64, 4, [1, 90, 3], [208, 300, 105]),
    (7, 2, 256, 4, [40, 1], [300, 13]),
]


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("P,H,D,Hq,q_len,kv_len", ODD_PAGES)
def test_pages_of_other_sizes(cache, P, H, D, Hq, q_len, kv_len):
    check(Paged(90, P, H, D, cache, q_len, kv_len).fill(spread=1).up(), Hq)


MISSING = [  # P, H, D, Hq, rows
    (16, 2, 64, 4, 1), (16, 2, 64, 4, 60),
    (104, 1, 64, 4, 1), (104, 1, 64, 4, 60),
    (104, 1, 128, 4, 1), (104, 1, 128, 4, 20), (104, 1, 128, 4, 80),
    (16, 2, 128, 4, 30),
    (16, 1, 256, 6, 1), (16, 1, 256, 6, 40),
    (104, 1, 256, 6, 1), (104, 1, 256, 6, 40),
]


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("all_keys", [False, True])
@pytest.mark.parametrize("P,H,D,Hq,rows", MISSING)
def test_missing_pages(cache, P, H, D, Hq, rows, all_keys):
    kv = [12 * P + 5, 7 * P - 3]
    c = Paged(91, P, H, D, cache, [rows, rows], kv).fill()
    c.table[0, [0, 3, 4, 9, 12]] = [-1, -1, c.n_pages, 2 ** 31 - 1, -(2 ** 31)]
    c.table[1, :] = -1  # nothing restored: zeros
    c.up()
    got = check(c, Hq, all_keys)
    assert not got[rows:].any() and got[:rows].any()


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("scale", [-0.125, 0.0, -0.0, 1.0, 2.0 ** -10, -3.0])
@pytest.mark.parametrize("H,D,Hq,q_len,kv_len", [
    (2, 64, 8, [1, 2], [300, 40]),
    (2, 64, 4, [60], [200]),
    (2, 128, 8, [1], [2000]),
    (2, 128, 4, [100, 1], [300, 77]),
    (1, 256, 6, [1], [200]),
    (1, 256, 6, [40], [200]),
])
def test_scales(cache, scale, H, D, Hq, q_len, kv_len):
    check(Paged(92, 16, H, D, cache, q_len, kv_len).fill().up(), Hq, scale=scale)
