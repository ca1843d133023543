"""The operators' binding refuses tensors whose elements are not what the kernels
read: integers and floats of torch's other sizes would be read as pairs."""
import pytest
import torch

from paper_2609_39358_amd import taliesin as T

FAKE = 0x10000  # an address that is never read


@pytest.mark.parametrize("dtype", [torch.int64, torch.int16, torch.float32, torch.float64])
@pytest.mark.parametrize("which,what", [(0, "row offsets"), (1, "cache lengths"), (2, "page tables")])
def test_batches(dtype, which, what):
    args = [FAKE] * 3
    args[which] = torch.zeros(64, dtype=dtype)
    with pytest.raises(ValueError, match="%s must be int32" % what):
        T.make_batch(1, 2, *args, 4)


@pytest.mark.parametrize("dtype", [torch.float64, torch.bfloat16, torch.int32])
def test_angles(dtype):
    with pytest.raises(ValueError, match="angles must be float32"):
        T.make_rope(torch.zeros(8, 32, 2, dtype=dtype), 64)


@pytest.mark.parametrize("dtype", [torch.int64, torch.float32])
def test_positions(dtype):
    with pytest.raises(ValueError, match="positions must be int32"):
        T.make_rope(torch.zeros(8, 32, 2, device="meta"), 64, torch.zeros(2, dtype=dtype))


def test_results():
    c = T.tl_ctx_create(b"tenant", b"model", 1, 2, 64, "bf16", 16)
    b, p = T.tl_batch(1, 2, FAKE, FAKE, FAKE, 4), T.tl_cache(FAKE, FAKE, c.slab_bytes, 4)
    x = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    for dtype in (torch.float64, torch.bfloat16):
        with pytest.raises(ValueError, match="lse must be float32"):
            T.tl_attend(c, None, 0, b, p, x, x, FAKE, 64, lse=torch.zeros(2, 2, dtype=dtype))
    with pytest.raises(ValueError, match="status must be uint8"):
        T.tl_append(c, None, 0, b, p, x, x, d_status=torch.zeros(2, dtype=torch.int32))


def test_types_that_are_taken():
    """What is refused next is that these are not on the device."""
    for dtype in (torch.int32, torch.uint32, torch.uint8):
        with pytest.raises(ValueError, match="device memory"):
            T.make_batch(1, 2, FAKE, torch.zeros(64, dtype=dtype), FAKE, 4)
    with pytest.raises(ValueError, match="device memory"):
        T.make_rope(torch.zeros(8, 32, 2), 64)
