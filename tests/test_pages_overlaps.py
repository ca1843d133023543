"""Calls on pages and kept rows whose results lie over something else that they are given
are refused, whichever arrays these are; neighbours that touch are not."""
import ctypes
import itertools

import pytest

from paper_2609_39358_amd import taliesin as T
from tests.test_operators_host import FAKE, cache, ctx

N, PARENTS, WIDTH, PAGES, GROUPS, ROWS = 12, 3, 5, 40, 2, 31
CTX = dict(layers=2, layer_group=[0, 1])


def fork_arrays(c):
    row = 4 * GROUPS * WIDTH
    need = T.tl_pages_workspace_bytes(c, N, PAGES)
    return (dict(refs=4 * GROUPS * PAGES, tables_out=N * row, len_out=4 * N, status=N, ws=need),
            dict(kv_len=4 * PARENTS, tables=PARENTS * row, parent=4 * N))


def fork(c, a, n=N):
    p = T.tl_pool(a["refs"], PAGES)
    return T.lib().tl_pages_fork(c.handle, None, ctypes.byref(p), ctypes.byref(cache(c, n_pages=PAGES)), PARENTS, a["kv_len"], a["tables"], n, a["parent"],
                                 a["len_out"], a["tables_out"], WIDTH, a["status"], a["ws"], 0)


def take_arrays(c):
    return (dict(refs=4 * GROUPS * PAGES, tables=4 * GROUPS * N * WIDTH, status=N, ws=T.tl_pages_workspace_bytes(c, N, PAGES)), dict(have=4 * N, want=4 * N))


def take(c, a, n=N):
    p = T.tl_pool(a["refs"], PAGES)
    return T.lib().tl_pages_take(c.handle, None, ctypes.byref(p), n, a["have"], a["want"], a["tables"], WIDTH, a["status"], a["ws"], 0)


def free_arrays(c):
    return dict(refs=4 * GROUPS * PAGES, tables=4 * GROUPS * N * WIDTH), dict(first=4 * N, end=4 * N)


def free(c, a, n=N):
    p = T.tl_pool(a["refs"], PAGES)
    return T.lib().tl_pages_free(c.handle, None, ctypes.byref(p), n, a["tables"], WIDTH, a["first"], a["end"])


def keep_arrays(c):
    return dict(len_out=4 * N, status=N), dict(kv_len=4 * N, row_off=4 * N + 4, n_keep=4 * N, keep=4 * ROWS, tables=4 * GROUPS * N * WIDTH)


def keep(c, a, n=N):
    b = T.tl_batch(n, ROWS, a["row_off"], a["kv_len"], a["tables"], WIDTH)
    return T.lib().tl_keep(c.handle, None, ctypes.byref(b), a["n_keep"], a["keep"], ctypes.byref(cache(c, n_pages=PAGES)), a["len_out"], a["status"])


CALLS = [(fork, fork_arrays), (take, take_arrays), (free, free_arrays), (keep, keep_arrays)]


def laid_out(sizes):
    """Addresses far apart."""
    return {name: FAKE + (i + 1 << 32) for i, name in enumerate(sizes)}


@pytest.mark.parametrize("call,arrays", CALLS)
def test_results_over_other_arrays(call, arrays):
    c = ctx(**CTX)
    written, read = arrays(c)
    sizes = {**written, **read}
    for a, b in itertools.permutations(sizes, 2):
        if a in read and b in read:
            continue
        step = 16 if "ws" in (a, b) else 4
        for at in (0, (sizes[b] - 1) // step * step, step):  # its begin, its last whole step, in it
            if at >= sizes[b]:
                continue
            where = laid_out(sizes)
            where[a] = where[b] + at
            if a != "ws" or where[a] % 16 == 0:
                assert call(c, where) == T.TL_EINVAL, (a, b, at)


@pytest.mark.parametrize("call,arrays", [x for x in CALLS if x[0] in (fork, take)])
def test_neighbours(call, arrays):
    """(A workspace of no bytes is refused behind these checks: nothing is enqueued.)"""
    c = ctx(**CTX)
    written, read = arrays(c)
    sizes = {**written, **read}
    assert call(c, laid_out(sizes)) == T.TL_ERANGE
    for a, b in itertools.permutations(sizes, 2):
        where = laid_out(sizes)
        where[a] = where[b] + -(-sizes[b] // 16) * 16
        assert call(c, where) == T.TL_ERANGE, (a, b)
        if a in read and b in read:  # these may share
            where[a] = where[b]
            assert call(c, where) == T.TL_ERANGE, (a, b)
    if call is fork:
        assert call(c, dict(laid_out(sizes), status=None)) == T.TL_ERANGE


@pytest.mark.parametrize("call,arrays", CALLS)
def test_nothing_to_do(call, arrays):
    written, read = arrays(ctx(**CTX))
    assert call(ctx(**CTX), {name: FAKE for name in {**written, **read}}, n=0) == T.TL_OK
