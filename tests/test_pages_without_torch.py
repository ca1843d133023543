"""The calls on pages and kept rows from a program that has no torch: addresses and numpy
arrays are taken as the C ABI takes them, and refusals are the library's."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
import sys
sys.modules["torch"] = None  # import torch raises ImportError
import numpy as np
from paper_2609_39358_amd import taliesin as T

A = [0x10000 + (i << 32) for i in range(9)]  # addresses that are never read
c = T.tl_ctx_create(b"tenant", b"model", 2, 2, 64, "bf16", 16)
pages = T.tl_cache(A[0], A[0], c.slab_bytes, 4)
pool = T.make_pool(A[1], 4)
ws = 1 << 40


def calls(n, odd=0):
    batch = T.make_batch(n, 0, A[2] + odd, A[3], A[4], 4)
    return (
        lambda: T.tl_pages_copy(c, None, pages, n, A[2] + odd, A[3], A[4]),
        lambda: T.tl_pages_fork(c, None, pool, pages, 2, A[2] + odd, A[3], n, A[4], A[5], A[6], 4, A[7], ws, None),
        lambda: T.tl_pages_take(c, None, pool, n, A[2], A[3] + odd, A[4], 4, A[7], ws, A[8]),
        lambda: T.tl_pages_free(c, None, pool, n, A[2] + odd, 4, A[3], None),
        lambda: T.tl_keep(c, None, batch, pages, A[5], A[6], A[7], A[8]),
    )


for call in calls(0):  # nothing to do
    call()
T.tl_pages_free(c, None, pool, 0, np.zeros(4, np.int32), 4)
for i, call in enumerate(calls(3, 1)):  # not on a word
    try:
        call()
    except T.TaliesinError as e:
        assert e.status == T.TL_EINVAL, (i, e.status)
    else:
        raise AssertionError(i)
print("done")
"""


def test_addresses():
    run = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip().endswith("done"), run.stdout
