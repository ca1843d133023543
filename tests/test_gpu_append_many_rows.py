"""The largest batches of rows that tl_append takes."""
import numpy as np
import pytest
import torch

from paper_2609_39358_amd import taliesin as T
from paper_2609_39358_amd.device import PagedCache
from tests.paged_case import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache,P", [("fp8_scaled", 1), ("fp8_scaled", 16), ("bf16", 16)])
def test_as_many_rows_as_a_batch_has(cache, P):
    """2^24 - 1 rows of one request: one row, read again and again, into the few pages that there are."""
    H, D, n = 1, 64, (1 << 24) - 1
    ctx = T.tl_ctx_create(b"tenant", b"model", 1, H, D, cache, P)
    pages = PagedCache(1, 4, ctx.slab_bytes, DEV).zero_()
    x = torch.ones((1, H, D), dtype=torch.bfloat16, device=DEV).expand(n, H, D)
    width = -(-n // P)
    table = torch.full((1, 1, width), -1, dtype=torch.int32, device=DEV)
    named = {0: 2, width // 2: 0, width - 1: 3}
    for at, page in named.items():
        table[0, 0, at] = page
    off, kv = torch.tensor([0, n], dtype=torch.int32, device=DEV), torch.tensor([n], dtype=torch.int32, device=DEV)
    status = torch.zeros(n, dtype=torch.uint8, device=DEV)
    T.tl_append(ctx, None, 0, T.make_batch(1, n, off, kv, table, width), pages.tl(), x, x, d_status=status)
    got = np.flatnonzero(status.cpu().numpy() == T.ACCEPT)
    want = np.concatenate([np.arange(at * P, min(at * P + P, n)) for at in sorted(named)])
    assert np.array_equal(got, want)
    assert int((status == T.BADARG).sum()) == n - want.size
    bytes_of = P * H * D * (2 if cache == "bf16" else 1)
    for k in (pages.k[0], pages.v[0]):
        k = k.cpu().numpy()
        assert not k[1].any()
        for page in named.values():
            rows = n - (width - 1) * P if page == 3 else P
            codes = k[page, :bytes_of].reshape(P, -1)[:rows]
            assert (codes == codes[0]).all() and codes.any()
