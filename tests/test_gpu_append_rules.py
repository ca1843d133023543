"""tl_append on both sides of the sizes where windows of rows become shorter and heads go to
other numbers of workgroups: byte for byte, as in test_gpu_append, and with norms."""
import pytest

from tests.test_gpu_append import test_append as appended
from tests.test_gpu_norm import test_heads_of_one_magnitude as normed

pytestmark = pytest.mark.gpu

SIDES = [  # P, H, D, q_len, held
    (16, 8, 128, [900], 0),           # so few fragments that windows become shorter
    (16, 8, 128, [1100], 5),
    (128, 3, 64, [128 * 126], 3),     # long ones of few heads, and one window more than that
    (128, 3, 64, [128 * 129], 3),
    (128, 8, 64, [300] * 34, 50),     # long ones of several requests
    (256, 16, 64, [500] * 20, 9),
    (256, 16, 64, [500] * 28, 9),
    (16, 8, 64, [24] * 100, 7),       # requests longer than a page
    (16, 8, 64, [24] * 175, 7),
    (16, 16, 64, [16] * 100, 7),      # and no longer
    (16, 16, 64, [5] * 300, 3),       # heads of which a workgroup takes four, or all, at once
    (16, 16, 64, [2] * 520, 3),
    (16, 8, 128, [1 + i * 7 % 24 for i in range(96)], 5),   # lengths that differ
    (64, 8, 128, [1 + i * 11 % 50 for i in range(40)], 9),
    (16, 4, 256, [1 + i * 5 % 14 for i in range(130)], 1),
]


def place(q_len, held, P):
    return [n + (held * (i + 1)) % (2 * P) for i, n in enumerate(q_len)]


@pytest.mark.parametrize("P,H,D,q_len,held", SIDES)
def test_append(P, H, D, q_len, held):
    appended("fp8_scaled", P, H, D, H, D, 1, False, q_len, place(q_len, held, P), 0)


@pytest.mark.parametrize("P,H,D,q_len,held", [x for x in SIDES if sum(x[3]) < 6000])
def test_append_with_norms(P, H, D, q_len, held):
    normed("fp8_scaled", True, True, P, H, D, H, D, 1, False, q_len, place(q_len, held, P), 0)
