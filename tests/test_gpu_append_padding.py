"""Rows that no request owns (a captured step's padding) keep what q_out holds there,
but for rows that positions of the caller's own turn."""
import numpy as np
import pytest
import torch

from paper_2609_39358_amd import taliesin as T
from tests import paged_case as pc
from tests.paged_case import DEV, Paged
from tests.test_gpu_append import angles, make_rows, same_bf16, same_pages

pytestmark = pytest.mark.gpu

PAD = 5


@pytest.mark.parametrize("cache", ["bf16", "fp8_scaled"])
@pytest.mark.parametrize("rotated", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_padding_rows_are_left_alone(cache, rotated, in_place):
    P, H, D, Hq = 16, 2, 64, 4
    c = Paged(60, P, H, D, cache, [3, 0, 20], [7, 4, 33]).fill().up()
    rows = c.rows + PAD
    x, host = make_rows(c.r, rows, Hq + 2 * H, D)
    d = x.to(DEV)
    q_out = d[:, :Hq] if in_place else torch.full((rows, Hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    cs = angles(33, D // 2)
    rope = T.make_rope(torch.from_numpy(cs).to(DEV), D) if rotated else None
    status = torch.zeros(rows, dtype=torch.uint8, device=DEV)
    T.tl_append(c.ctx, None, 0, c.batch(rows), c.paged.tl(), d[:, Hq:Hq + H], d[:, Hq + H:], rope, d[:, :Hq], q_out, status)
    n, pos = c.rows, np.concatenate([np.arange(4, 7), np.arange(13, 33)])[None]
    turn = (lambda y: pc.rotate(y, cs, pos, [0] * (D // 2), D, False)) if rotated else (lambda y: y)
    pc.append(c, turn(host[:n, Hq:Hq + H]), host[:n, Hq + H:])
    same_pages(c)
    same_bf16(q_out[:n], turn(host[:n, :Hq]))
    same_bf16(q_out[n:], host[n:, :Hq] if in_place else np.full((PAD, Hq, D), 7.0, np.float32))
    same_bf16(d[:, Hq:], host[:, Hq:])
    assert np.array_equal(status.cpu().numpy(), [T.ACCEPT] * n + [T.BADARG] * PAD)


def test_padding_rows_with_positions():
    """Turned where their position has an angle, left alone where it has none."""
    P, H, D, Hq = 16, 2, 64, 4
    c = Paged(61, P, H, D, "fp8_scaled", [3], [7]).fill().up()
    rows = c.rows + PAD
    x, host = make_rows(c.r, rows, Hq + 2 * H, D)
    d = x.to(DEV)
    pos = np.array([4, 5, 6, 9, -1, 33, 0, -(2 ** 31)], np.int32)
    cs = angles(33, D // 2)
    rope = T.make_rope(torch.from_numpy(cs).to(DEV), D, torch.from_numpy(pos).to(DEV))
    q_out = torch.full((rows, Hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    T.tl_append(c.ctx, None, 0, c.batch(rows), c.paged.tl(), d[:, Hq:Hq + H], d[:, Hq + H:], rope, d[:, :Hq], q_out)
    angle = (pos >= 0) & (pos < 33)
    want = pc.rotate(host[:, :Hq], cs, np.where(angle, pos, 0)[None], [0] * (D // 2), D, False)
    want[~angle] = 7.0
    same_bf16(q_out, want)
