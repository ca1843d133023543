"""tl_append where a window's heads go to several workgroups, and where long pages' windows
are shorter than their fragments: byte for byte, as in test_gpu_append."""
import pytest

from tests.test_gpu_append import test_append as appended

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H", [1, 5, 16])
@pytest.mark.parametrize("P,D,q_len,held", [
    (256, 128, [500, 500, 300], 0),     # a few long fragments
    (256, 64, [1000], 77),
    (104, 256, [250, 3, 90, 104], 60),
    (65, 64, [65] * 5, 0),              # one row more than a window
    (64, 128, [64] * 5, 1),
    (16, 64, [1, 24, 7, 13, 2, 19], 11),  # drafts
    (16, 128, [9] * 40, 3),
    (16, 256, [4] * 90, 14),
    (16, 128, [2] * 3, 15),
])
def test_heads_on_several_workgroups(H, P, D, q_len, held):
    appended("fp8_scaled", P, H, D, H, D, 1, False, q_len, [n + (held * (i + 1)) % (2 * P) for i, n in enumerate(q_len)], 0)
