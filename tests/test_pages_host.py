"""tl_pages_* and tl_keep on the host: what is refused before anything is enqueued,
by the library and by the binding, and the workspace's size."""
import ctypes

import pytest
import torch

from paper_2609_39358_amd import taliesin as T
from tests.test_operators_host import FAKE, batch, cache, ctx

FAR = FAKE + (1 << 30)  # addresses of their own
LENS, OUT, PARENT, TABLES, STATUS, WS = (FAKE + (i << 32) for i in range(1, 7))
BIG = 1 << 50


def ref(x):
    return None if x is None else ctypes.byref(x)


def pool(**kw):
    a = dict(d_refs=FAKE, n_pages=4)
    a.update(kw)
    return T.tl_pool(**a)


def copy(c, pages=None, n=3, src=FAKE, dst=FAR, rows=None):
    return T.lib().tl_pages_copy(c.handle, None, ref(pages or cache(c)), n, src, dst, rows)


def fork(c, p=None, pages=None, n_parents=2, kv_len=LENS, tables=TABLES, n=3, parent=PARENT, len_out=OUT, tables_out=FAR, width=4, ws=WS, size=BIG):
    return T.lib().tl_pages_fork(c.handle, None, ref(p or pool()), ref(pages or cache(c)), n_parents, kv_len, tables, n, parent, len_out, tables_out,
                                 width, None, ws, size)


def take(c, p=None, n=3, have=LENS, want=OUT, tables=TABLES, width=4, ws=WS, size=BIG):
    return T.lib().tl_pages_take(c.handle, None, ref(p or pool()), n, have, want, tables, width, None, ws, size)


def free(c, p=None, n=3, tables=TABLES, width=4, first=None, end=None):
    return T.lib().tl_pages_free(c.handle, None, ref(p or pool()), n, tables, width, first, end)


def keep(c, b=None, n_keep=PARENT, rows=TABLES, pages=None, len_out=OUT, status=None):
    return T.lib().tl_keep(c.handle, None, ref(b or batch()), n_keep, rows, ref(pages or cache(c)), len_out, status)


PAGES = [(dict(d_layer_k=None), T.TL_EINVAL), (dict(d_layer_v=FAKE + 4), T.TL_EINVAL), (dict(page_stride=2048), T.TL_EINVAL),
         (dict(page_stride=4104), T.TL_EINVAL), (dict(n_pages=-1), T.TL_EINVAL), (dict(n_pages=1 << 31), T.TL_EINVAL)]


@pytest.mark.parametrize("call", [copy, fork, keep])
@pytest.mark.parametrize("kw,status", PAGES)
def test_caches(call, kw, status):
    c = ctx()
    assert call(c, pages=cache(c, **kw)) == status


@pytest.mark.parametrize("call", [fork, take, free])
@pytest.mark.parametrize("kw", [dict(d_refs=None), dict(d_refs=FAKE + 2), dict(n_pages=-1), dict(n_pages=1 << 31)])
def test_pools(call, kw):
    assert call(ctx(), p=pool(**kw)) == T.TL_EINVAL


@pytest.mark.parametrize("call", [fork, take, free])
@pytest.mark.parametrize("kw", [dict(n=1 << 20), dict(width=1 << 28), dict(n=1 << 12, width=1 << 19)])
def test_sizes(call, kw):
    assert call(ctx(), **kw) == T.TL_ERANGE


@pytest.mark.parametrize("kw,status", [
    (dict(src=None), T.TL_EINVAL), (dict(dst=FAR + 1), T.TL_EINVAL), (dict(rows=FAKE + 2), T.TL_EINVAL), (dict(n=1 << 24), T.TL_ERANGE),
    (dict(n=0, src=None, dst=None), T.TL_OK)])
def test_copy(kw, status):
    assert copy(ctx(), **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(kv_len=None), T.TL_EINVAL), (dict(kv_len=LENS + 1), T.TL_EINVAL), (dict(tables=None), T.TL_EINVAL), (dict(parent=None), T.TL_EINVAL),
    (dict(len_out=None), T.TL_EINVAL), (dict(tables_out=None), T.TL_EINVAL), (dict(ws=None), T.TL_EINVAL), (dict(ws=WS + 8), T.TL_EINVAL),
    (dict(tables_out=TABLES), T.TL_EINVAL), (dict(tables_out=TABLES + 2 * 4 * 4 - 4), T.TL_EINVAL), (dict(tables_out=TABLES - 3 * 4 * 4 + 4), T.TL_EINVAL),
    (dict(len_out=LENS + 4), T.TL_EINVAL), (dict(len_out=PARENT), T.TL_EINVAL), (dict(p=pool(n_pages=3)), T.TL_EINVAL),
    (dict(n_parents=1 << 20), T.TL_ERANGE), (dict(n=0, parent=None, len_out=None), T.TL_OK)])
def test_fork(kw, status):
    assert fork(ctx(), **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(have=None), T.TL_EINVAL), (dict(want=OUT + 2), T.TL_EINVAL), (dict(tables=None), T.TL_EINVAL), (dict(ws=None), T.TL_EINVAL),
    (dict(n=0, have=None, want=None), T.TL_OK)])
def test_take(kw, status):
    assert take(ctx(), **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(tables=None), T.TL_EINVAL), (dict(tables=TABLES + 1), T.TL_EINVAL), (dict(first=LENS + 1), T.TL_EINVAL), (dict(end=LENS + 2), T.TL_EINVAL),
    (dict(n=0, tables=None), T.TL_OK), (dict(width=0, tables=None), T.TL_OK)])
def test_free(kw, status):
    assert free(ctx(), **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(n_keep=None), T.TL_EINVAL), (dict(rows=None), T.TL_EINVAL), (dict(rows=TABLES + 1), T.TL_EINVAL), (dict(len_out=None), T.TL_EINVAL),
    (dict(len_out=FAKE), T.TL_EINVAL), (dict(len_out=PARENT), T.TL_EINVAL), (dict(b=batch(d_row_off=None)), T.TL_EINVAL),
    (dict(len_out=TABLES + 4), T.TL_EINVAL), (dict(b=batch(d_row_off=OUT - 4)), T.TL_EINVAL),
    (dict(b=batch(n_rows=0, d_kv_len=None)), T.TL_EINVAL), (dict(b=batch(d_tables=None)), T.TL_EINVAL), (dict(b=batch(n_rows=1 << 24)), T.TL_ERANGE),
    (dict(b=batch(n_reqs=1 << 20)), T.TL_ERANGE), (dict(b=batch(n_reqs=0, d_row_off=None), n_keep=None), T.TL_OK)])
def test_keep(kw, status):
    assert keep(ctx(), **kw) == status


def test_keep_takes_the_values_that_the_operators_take():
    assert keep(ctx("f16")) == keep(ctx(D=32)) == T.TL_ELAYOUT


def test_workspace():
    """Room for a number and a status for each request and for a page's id of each page, in each group."""
    c = ctx(layers=2, layer_group=[0, 1])
    for n, pages in ((0, 0), (1, 1), (255, 70000), (4096, 12)):
        assert 2 * 4 * (n + 1 + pages) + n <= T.tl_pages_workspace_bytes(c, n, pages) <= 2 * 4 * (n + 1 + pages) + n + 1024
        assert T.tl_pages_workspace_bytes(c, n, pages) <= T.tl_pages_workspace_bytes(c, n + 1, pages + 1)
    need = T.tl_pages_workspace_bytes(c, 3, 4)
    assert fork(c, size=need - 1) == take(c, size=need - 1) == T.TL_ERANGE


@pytest.mark.parametrize("dtype", [torch.int64, torch.float32])
def test_types(dtype):
    c = ctx()
    x, p, b = torch.zeros(64, dtype=dtype), pool(), batch()
    for what, call in (("page counts", lambda: T.make_pool(x)),
                       ("source pages", lambda: T.tl_pages_copy(c, None, cache(c), 2, x, FAKE)),
                       ("rows", lambda: T.tl_pages_copy(c, None, cache(c), 2, FAKE, FAKE, x)),
                       ("parents", lambda: T.tl_pages_fork(c, None, p, cache(c), 2, LENS, TABLES, 3, x, OUT, FAR, 4, WS, BIG)),
                       ("lengths", lambda: T.tl_pages_take(c, None, p, 3, LENS, x, TABLES, 4, WS, BIG)),
                       ("page tables", lambda: T.tl_pages_free(c, None, p, 3, x, 4)),
                       ("kept rows", lambda: T.tl_keep(c, None, b, cache(c), FAKE, x, OUT))):
        with pytest.raises(ValueError, match="%s must be int32" % what):
            call()
    with pytest.raises(ValueError, match="status must be uint8"):
        T.tl_keep(c, None, b, cache(c), FAKE, FAKE, OUT, torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="device memory"):
        T.tl_pages_free(c, None, p, 3, torch.zeros(12, dtype=torch.int32), 4)
