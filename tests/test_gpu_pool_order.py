"""Who is served by tl_pages_take and tl_pages_fork where a pool runs short, as the header
has it: each request is meant to have the lowest free pages behind those of the requests
before it, a refused one takes nothing, and nobody overtakes it, in any group of layers."""
import numpy as np
import pytest
import torch

from paper_2609_39358_amd import taliesin as T
from tests.pages_case import DEV, Pages, up

pytestmark = pytest.mark.gpu

P = 16


def take(groups, n_pages, used, want, width, tables=None):
    """[n] requests that have nothing and want want[i] pages (tokens: want[i] * P). (status, tables, counts)"""
    c = Pages(1, P, 1, 64, "fp8", 1, len(groups), groups).up()
    n = len(want)
    refs = np.zeros((c.groups, n_pages), np.int32)
    for g, pages in enumerate(used):
        refs[g, pages] = 1
    tables = np.full((c.groups, n, width), -1, np.int32) if tables is None else tables
    d_refs, d_tables = up(refs), up(tables)
    size = T.tl_pages_workspace_bytes(c.ctx, n, n_pages)
    ws, status = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV), torch.full((n,), 77, dtype=torch.uint8, device=DEV)
    T.tl_pages_take(c.ctx, None, T.make_pool(d_refs), n, up(np.zeros(n)), up(np.array(want) * P), d_tables, width, ws, size, status)
    torch.cuda.synchronize()
    return status.tolist(), d_tables.cpu().numpy(), d_refs.cpu().numpy()


def test_a_large_request_is_not_overtaken():
    status, tables, refs = take([0], 12, [[0, 5, 7]], [2, 10, 1, 0, 1], 10)
    assert status == [T.ACCEPT, T.MISSING, T.MISSING, T.ACCEPT, T.MISSING]
    assert tables[0, 0].tolist() == [1, 2] + [-1] * 8 and (tables[0, 1:] == -1).all()
    assert refs[0].tolist() == [1, 1, 1, 0, 0, 1, 0, 1, 0, 0, 0, 0]


def test_named_last_it_stops_nobody():
    status, tables, refs = take([0], 12, [[0, 5, 7]], [2, 1, 0, 1, 10], 10)
    assert status == [T.ACCEPT] * 4 + [T.MISSING]
    assert tables[0, :4, 0].tolist() == [1, 3, -1, 4] and (tables[0, 4] == -1).all()


def test_one_past_its_row_wants_none():
    status, tables, _ = take([0], 4, [[]], [3, 9, 1], 3)
    assert status == [T.ACCEPT, T.BADARG, T.ACCEPT]
    assert tables[0].tolist() == [[0, 1, 2], [-1] * 3, [3, -1, -1]]


@pytest.mark.parametrize("many", [0, 1500])
def test_what_is_meant_for_a_refused_request_stays_free_in_every_group(many):
    """The second request is short in group 1 alone; the third wants pages of group 0 only,
    and is given those behind the second's. (many: requests that want nothing before them, more than a
    thread each.)"""
    n = many + 4
    tables = np.full((2, n, 3), -1, np.int32)
    tables[1, many + 2] = 9  # (has its pages there)
    want = [0] * many + [1, 3, 2, 1]
    status, t, refs = take([0, 1], 12, [[], range(3, 12)], want, 3, tables)
    assert status[:many] == [T.ACCEPT] * many
    assert status[many:] == [T.ACCEPT, T.MISSING, T.ACCEPT, T.MISSING]
    assert t[0, many:].tolist() == [[0, -1, -1], [-1] * 3, [4, 5, -1], [-1] * 3]
    assert t[1, many:].tolist() == [[0, -1, -1], [-1] * 3, [9, 9, 9], [-1] * 3]
    assert refs[0].nonzero()[0].tolist() == [0, 4, 5] and refs[1].nonzero()[0].tolist() == [0] + list(range(3, 12))


def test_branches():
    """Branches want a page where their parent's last one is partly filled, in the groups that
    name it: the second is short in group 1, the third wants a page of group 0 alone."""
    c = Pages(2, P, 2, 64, "bf16", 8, 2, [0, 1]).up()
    refs = np.ones((2, 8), np.int32)
    refs[0, 4:8] = 0
    refs[1, 5] = 0
    kv = np.array([P + 3, P + 3])
    tables = np.array([[[0, 1], [2, 3]], [[0, 1], [2, -1]]], np.int32)  # parent 1's last page is not there in group 1
    parent, n = np.array([0, 0, 1, 0]), 4
    d_refs, out, lens = up(refs), torch.full((2, n, 2), 77, dtype=torch.int32, device=DEV), up(np.zeros(n))
    status = torch.full((n,), 77, dtype=torch.uint8, device=DEV)
    size = T.tl_pages_workspace_bytes(c.ctx, n, 8)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV)
    T.tl_pages_fork(c.ctx, None, T.make_pool(d_refs), c.paged.tl(), 2, up(kv), up(tables), n, up(parent), lens, out, 2, ws, size, status)
    torch.cuda.synchronize()
    assert status.tolist() == [T.ACCEPT, T.MISSING, T.ACCEPT, T.MISSING] and lens.tolist() == [P + 3, 0, P + 3, 0]
    assert out[0].tolist() == [[0, 4], [-1, -1], [2, 6], [-1, -1]]
    assert out[1].tolist() == [[0, 5], [-1, -1], [2, -1], [-1, -1]]
    assert d_refs.tolist() == [[2, 1, 2, 1, 1, 0, 1, 0], [2, 1, 2, 1, 1, 1, 1, 1]]
    for page, where in ((4, 1), (6, 3)):  # copies of the last page's three rows
        rows = 3 * c.row
        c.host[:2, page, :rows] = c.host[:2, where, :rows]
    c.host[2:, 5, :3 * c.row] = c.host[2:, 1, :3 * c.row]
    c.same()
