"""tl_append_norm on the host: what is refused before anything is enqueued."""
import ctypes

import pytest
import torch

from paper_2609_39358_amd import taliesin as T
from tests.test_operators_host import FAKE, batch, cache, ctx, rows


def norm(**kw):
    a = dict(d_q_weight=FAKE, d_k_weight=FAKE, q_stride=0, k_stride=64, eps=1e-6, flags=0)
    a.update(kw)
    return T.tl_norm(**a)


def call(c, n=None, b=None):
    return T.lib().tl_append_norm(c.handle, None, 0, ctypes.byref(b or batch()), None if n is None else ctypes.byref(n), None, ctypes.byref(rows()),
                                  ctypes.byref(rows()), 0, None, None, ctypes.byref(cache(c)), None)


@pytest.mark.parametrize("kw", [dict(d_q_weight=FAKE + 4), dict(d_k_weight=FAKE + 8), dict(q_stride=2), dict(k_stride=66), dict(k_stride=-(1 << 41)),
                                dict(q_stride=1 << 41), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=1e-39),
                                dict(flags=2)])
def test_refusals(kw):
    assert call(ctx(), norm(**kw)) == T.TL_EINVAL


def test_nothing_to_do():
    for n in (None, norm(), norm(d_q_weight=None, d_k_weight=None)):
        assert call(ctx(), n, batch(n_rows=0)) == T.TL_OK


def test_tensors():
    c = ctx()
    with pytest.raises(ValueError, match="norm weights must be float32"):
        T.make_norm(torch.ones(64, dtype=torch.bfloat16), None)
    with pytest.raises(ValueError, match="shape"):
        T.make_norm(torch.ones(1, 2, 64), None)
    with pytest.raises(ValueError, match="device memory"):
        T.make_norm(None, torch.ones(64))
    x = torch.zeros(2, 2, 64, dtype=torch.bfloat16)

    class OnDevice:  # stands for a device tensor: only its shape is asked for
        def __init__(self, *shape):
            self.shape = shape

        def dim(self):
            return len(self.shape)

    for shape in ((32,), (3, 64), (2, 128)):
        n = norm()
        n._keep = (None, OnDevice(*shape))
        with pytest.raises(ValueError, match="norm weights .* for 2 heads of 64"):
            T._check_norm(n, 64, (0, 2))
    with pytest.raises(ValueError, match="device memory"):
        T.tl_append(c, None, 0, batch(), cache(c), x, x, norm=norm())
