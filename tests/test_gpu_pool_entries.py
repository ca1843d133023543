"""tl_pages_take on tables whose entries name no page in other ways than -1: any id outside
[0, n_pages) is one that is wanted, as the other calls on pages have it."""
import numpy as np
import pytest
import torch

from paper_2609_39358_amd import taliesin as T
from tests.pages_case import DEV, Pages, up

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("width", [3, 70])  # walked by a lane, and by a wavefront
@pytest.mark.parametrize("groups", [[0], [0, 1]])
def test_ids_past_the_pool(width, groups):
    P, n, n_pages = 16, 5, 400
    c = Pages(1, P, 1, 64, "fp8", 1, len(groups), groups).up()
    refs = np.zeros((c.groups, n_pages), np.int32)
    refs[:, 0] = 1
    tables = np.full((c.groups, n, width), 0, np.int32)
    odd = [-1, n_pages, n_pages + 1, 2 ** 31 - 1, -2 ** 31]
    for i, x in enumerate(odd):
        tables[:, i, 1] = x
        tables[:, i, width - 1] = odd[i - 1]
    d_refs, d_tables = up(refs), up(tables)
    size = T.tl_pages_workspace_bytes(c.ctx, n, n_pages)
    ws, status = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV), torch.full((n,), 77, dtype=torch.uint8, device=DEV)
    T.tl_pages_take(c.ctx, None, T.make_pool(d_refs), n, up(np.zeros(n)), up(np.full(n, width * P)), d_tables, width, ws, size, status)
    torch.cuda.synchronize()
    for g in range(c.groups):
        for i in range(n):
            tables[g, i, 1], tables[g, i, width - 1] = 1 + 2 * i, 2 + 2 * i
    refs[:, :2 * n + 1] = 1
    assert status.tolist() == [T.ACCEPT] * n
    assert np.array_equal(d_tables.cpu().numpy(), tables) and np.array_equal(d_refs.cpu().numpy(), refs)
