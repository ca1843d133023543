"""tl_attend_tree on the host: what is refused before anything is enqueued."""
import ctypes

import pytest
import torch

from paper_2609_39358_amd import taliesin as T
from tests.test_operators_host import COMMON, FAKE, batch, cache, ctx, rows


def tree(**kw):
    a = dict(d_seen=FAKE, d_pos=FAKE, words=1)
    a.update(kw)
    return T.tl_tree(**a)


def attend(c, layer=0, b=None, t=None, heads=4, q=None, pages=None, scale=1.0, out=None, lse=None, ws=FAKE, ws_bytes=1 << 40, no_tree=False):
    return T.lib().tl_attend_tree(c.handle, None, layer, ctypes.byref(b or batch()), None if no_tree else ctypes.byref(t or tree()), heads,
                                  ctypes.byref(q or rows(row=256)), ctypes.byref(pages or cache(c)), scale, ctypes.byref(out or rows(row=256)), lse, ws, ws_bytes)


@pytest.mark.parametrize("kw,status", COMMON)
def test_what_tl_attend_refuses(kw, status):
    c = ctx()
    kw = dict(kw)
    if "pages" in kw:
        kw["pages"] = cache(c, **kw["pages"])
    assert attend(c, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(heads=3), T.TL_EINVAL), (dict(heads=0), T.TL_EINVAL), (dict(scale=float("inf")), T.TL_EINVAL), (dict(q=rows(FAKE + 8)), T.TL_EINVAL),
    (dict(out=rows(row=60)), T.TL_EINVAL), (dict(lse=FAKE + 2), T.TL_EINVAL), (dict(ws=None), T.TL_EINVAL), (dict(ws_bytes=100), T.TL_ERANGE)])
def test_other_arguments(kw, status):
    assert attend(ctx(), **kw) == status


@pytest.mark.parametrize("kw", [dict(d_seen=None), dict(d_seen=FAKE + 4), dict(d_pos=FAKE + 2), dict(words=0), dict(words=(1 << 18) + 1)])
def test_trees(kw):
    assert attend(ctx(), t=tree(**kw)) == T.TL_EINVAL


def test_a_window_asks_for_positions():
    assert attend(ctx(layer_window=[0, 100]), layer=1, t=tree(d_pos=None)) == T.TL_EINVAL


def test_no_tree_and_nothing_to_do():
    assert attend(ctx(), no_tree=True) == T.TL_EINVAL
    assert attend(ctx(), b=batch(n_rows=0)) == attend(ctx(), b=batch(n_reqs=0), t=tree(d_seen=None)) == T.TL_OK
    assert attend(ctx("f16")) == T.TL_ELAYOUT


def test_tensors():
    with pytest.raises(ValueError, match="masks must be int64"):
        T.make_tree(torch.zeros(4, 1, dtype=torch.int32))
    with pytest.raises(ValueError, match="positions must be int32"):
        T.make_tree(torch.zeros(4, 1, dtype=torch.int64), torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError, match="shape"):
        T.make_tree(torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError, match="device memory"):
        T.make_tree(torch.zeros(4, 1, dtype=torch.int64))
