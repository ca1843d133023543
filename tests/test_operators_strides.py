"""Results that overlap themselves are refused at any strides and numbers of rows."""
import ctypes

import pytest

from paper_2609_39358_amd import taliesin as T

FAKE = 0x10000  # an address that is never read: the workspace is too small for any call


def attend(rows, row, head, heads=2):
    c = T.tl_ctx_create(b"tenant", b"model", 1, 2, 64, "bf16", 16)
    b = T.tl_batch(1, rows, FAKE, FAKE, FAKE, 4)
    q, out, pages = T.tl_rows(FAKE, 128, 64), T.tl_rows(FAKE, row, head), T.tl_cache(FAKE, FAKE, c.slab_bytes, 4)
    return T.lib().tl_attend(c.handle, None, 0, ctypes.byref(b), heads, ctypes.byref(q), ctypes.byref(pages), 1.0, 0,
                             ctypes.byref(out), None, FAKE, 64)


@pytest.mark.parametrize("rows,row,head", [
    ((1 << 23) + 1, 1 << 40, (1 << 40) - 8),  # (rows - 1) * row is 2^63
    ((1 << 24) - 1, 1 << 40, (1 << 40) - 8),
    ((1 << 24) - 1, (1 << 40) - 8, 1 << 40),
    (2, 64, 64),
    (3, 128, 56),
    (3, 64, 128),
])
def test_overlapping(rows, row, head):
    assert attend(rows, row, head) == T.TL_EINVAL


@pytest.mark.parametrize("rows,row,head", [
    ((1 << 23) + 1, 1 << 40, 64),
    ((1 << 24) - 1, 1 << 40, 1 << 39),
    ((1 << 15), 64, 1 << 40),
    (2, 128, 64),
    (2, 64, 128),
    (1, 0, 64),
])
def test_apart(rows, row, head):
    assert attend(rows, row, head) == T.TL_ERANGE  # of the workspace, which is looked at last
