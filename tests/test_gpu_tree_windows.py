"""tl_attend with a tree on layers whose windows are on both sides of the size up to which a
tile goes to one workgroup as a whole, where one request is longer than the window and the
others are short: against 64 bits, as in test_gpu_tree."""
import numpy as np
import pytest

from tests.paged_case import Paged
from tests.test_gpu_tree import check, trees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("window", [1900, 2044, 2100, 30000])
@pytest.mark.parametrize("H,D,Hq,n,new", [
    (16, 64, 16, 64, 4),    # 32 rows a wavefront
    (16, 128, 16, 60, 4),
    (8, 128, 32, 16, 34),   # tiles of many rows
    (8, 256, 8, 20, 20),
])
def test_one_long_request(cache, window, H, D, Hq, n, new):
    r = np.random.default_rng(19)
    before = r.integers(0, 60, n)
    before[n // 3] = min(window + 70, 2700)
    c = Paged(20, 16, H, D, cache, [new] * n, [new + int(b) for b in before], window=window).fill(spread=1).up()
    see, depth = trees(c, r, 3)
    check(c, Hq, see, depth, 1)
