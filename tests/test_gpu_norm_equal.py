"""tl_append with centred norms of heads whose elements are all equal, or all but one: what
is left of them is 0 exactly, or 64 bits' within the roundings, also where their sum or their
squares pass 32 bits."""
import numpy as np
import pytest
import torch

from paper_2609_39358_amd import taliesin as T
from tests.paged_case import DEV, Paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_equal_elements(cache, D):
    """The largest finite value, values whose sum or whose squares alone are too large, and
    others: (x - mean) is 0, and 0 / sqrt(0 + eps) is 0."""
    values = [3.38e38, -3.38e38, 2.0 ** 127, 2.0 ** 121, 2.0 ** 120 * 1.9921875, 2.0 ** 70, 1.0, -2.0 ** -100, 0.0]
    n = len(values)
    c = Paged(1, 16, 2, D, cache, [n], [n + 3]).fill().up()
    x = torch.tensor(values, device=DEV).to(torch.bfloat16)[:, None, None].expand(n, 6, D).contiguous()
    assert x.isfinite().all()
    w = torch.linspace(-2, 2, D, device=DEV)
    q = torch.full_like(x[:, :2], 7.0)
    T.tl_append(c.ctx, None, 0, c.batch(), c.paged.tl(), x[:, 2:4], x[:, 4:], None, x[:, :2], q, norm=T.make_norm(w, w, 1e-6, True))
    torch.cuda.synchronize()
    c.pages = [c.dk.cpu().numpy(), c.dv.cpu().numpy()]
    assert not q.float().any()
    assert not np.any(c.values(0, 0)[3:])


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("big", [3.38e38, 2.0 ** 121, 2.0 ** 65])
def test_all_but_one(D, big):
    """Of D equal elements the first is 0 or has the other sign. Less their mean the others are
    a / D and 2 a / D of it, and the first D - 1 times as much: 1 / sqrt(D - 1) and -sqrt(D - 1)
    after the norm. Each mean, difference, sum, product, root and quotient is off by 2^-24 at
    most, the mean against a D-th part of its size: 2^-24 * D * 8 in all, and half a step of
    bf16 for the result."""
    c = Paged(2, 16, 2, D, "bf16", [2], [2]).fill().up()
    x = torch.full((2, 6, D), big, device=DEV)
    x[0, :, 0], x[1, :, 0] = 0, -big
    x = x.to(torch.bfloat16)
    q = torch.empty_like(x[:, :2])
    T.tl_append(c.ctx, None, 0, c.batch(), c.paged.tl(), x[:, 2:4], x[:, 4:], None, x[:, :2], q, norm=T.make_norm(None, None, 1e-6, True))
    want = torch.full((D,), (D - 1) ** -0.5, dtype=torch.float64)
    want[0] = -(D - 1) ** 0.5
    off = want.abs() * (2.0 ** -8 + D * 8 * 2.0 ** -24)
    assert ((q.cpu().double() - want).abs() <= off).all()
