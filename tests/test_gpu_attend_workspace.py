"""One workspace, made for the largest batch, serves the smaller ones."""
import numpy as np
import pytest
import torch

from paper_2609_39358_amd import taliesin as T
from tests import paged_case as pc
from tests.paged_case import DEV, Paged
from tests.test_gpu_attend import queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,D,Hq", [(2, 64, 8), (2, 128, 8), (1, 256, 6)])
def test_smaller_batches_in_a_workspace_made_for_the_largest(H, D, Hq):
    large = Paged(70, 16, H, D, "fp8_scaled", [1200], [1300])
    n = T.tl_attend_workspace_bytes(large.ctx, Hq, 8, 1200)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)
    for q_len in ([1], [4], [9], [20], [40], [5, 1], [1] * 8, [150, 30]):
        c = Paged(71, 16, H, D, "fp8_scaled", q_len, [m + 100 + 9 * i for i, m in enumerate(q_len)]).fill().up()
        d, q = queries(c, Hq)
        out = torch.empty((c.rows, Hq, D), dtype=torch.bfloat16, device=DEV)
        T.tl_attend(large.ctx, None, 0, c.batch(), c.paged.tl(), d, out, ws, n)
        want, _, tol, _ = pc.attend(c, q, D ** -0.5)
        assert (np.abs(out.float().cpu().numpy() - want) <= tol).all(), q_len
