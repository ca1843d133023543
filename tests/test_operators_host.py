"""tl_append, tl_attend and scaled 8-bit layouts on the host: what is refused
before anything is enqueued, the workspace sizes, the record geometry against the
oracle, and the number formats that the operator tests compare with."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import taliesin_ref as ref
from paper_2609_39358_amd import taliesin as T
from tests import paged_case as pc

FAKE = 0x10000  # an address that is never read: every call here is refused, or has nothing to do


def ctx(dtype="bf16", D=64, H=2, P=16, layers=2, **kw):
    return T.tl_ctx_create(b"tenant", b"model", layers, H, D, dtype, P, **kw)


def batch(**kw):
    a = dict(n_reqs=1, n_rows=2, d_row_off=FAKE, d_kv_len=FAKE, d_tables=FAKE, table_width=4)
    a.update(kw)
    return T.tl_batch(**a)


def rows(p=FAKE, row=2 * 64, head=64):
    return T.tl_rows(p, row, head)


def cache(c, **kw):
    a = dict(d_layer_k=FAKE, d_layer_v=FAKE, page_stride=c.slab_bytes, n_pages=4)
    a.update(kw)
    return T.tl_cache(**a)


AXIS = (ctypes.c_uint8 * 32)(*[0, 1] * 16)


def rope(**kw):
    a = dict(d_cos_sin=FAKE, n_angles=8, d_pos=None, rot_dim=64, n_axes=1, pair_axis=None, flags=0)
    a.update(kw)
    return T.tl_rope(**a)


def append(c, layer=0, b=None, r=None, k=None, v=None, heads=0, q=None, q_out=None, pages=None):
    ref_ = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
    return T.lib().tl_append(c.handle, None, layer, ref_(b or batch()), ref_(r), ref_(k or rows()), ref_(v or rows()), heads,
                             ref_(q), ref_(q_out), ref_(pages or cache(c)), None)


def attend(c, layer=0, b=None, heads=4, q=None, pages=None, scale=1.0, flags=0, out=None, lse=None, ws=FAKE, ws_bytes=1 << 40):
    return T.lib().tl_attend(c.handle, None, layer, ctypes.byref(b or batch()), heads, ctypes.byref(q or rows(row=256)),
                             ctypes.byref(pages or cache(c)), scale, flags, ctypes.byref(out or rows(row=256)), lse, ws, ws_bytes)


COMMON = [
    (dict(layer=2), T.TL_EINVAL),
    (dict(b=batch(d_row_off=None)), T.TL_EINVAL),
    (dict(b=batch(d_kv_len=None)), T.TL_EINVAL),
    (dict(b=batch(d_tables=None)), T.TL_EINVAL),
    (dict(b=batch(d_tables=FAKE + 2)), T.TL_EINVAL),
    (dict(b=batch(n_rows=1 << 24)), T.TL_ERANGE),
    (dict(b=batch(n_reqs=1 << 20)), T.TL_ERANGE),
    (dict(b=batch(table_width=1 << 28)), T.TL_ERANGE),
    (dict(pages=dict(d_layer_k=None)), T.TL_EINVAL),
    (dict(pages=dict(d_layer_v=FAKE + 4)), T.TL_EINVAL),
    (dict(pages=dict(page_stride=2048)), T.TL_EINVAL),
    (dict(pages=dict(page_stride=4104)), T.TL_EINVAL),
    (dict(pages=dict(n_pages=-1)), T.TL_EINVAL),
    (dict(pages=dict(n_pages=1 << 31)), T.TL_EINVAL),
]


@pytest.mark.parametrize("call", [append, attend])
@pytest.mark.parametrize("kw,status", COMMON)
def test_refusals_of_both(call, kw, status):
    c = ctx()
    kw = dict(kw)
    if "pages" in kw:
        kw["pages"] = cache(c, **kw["pages"])
    assert call(c, **kw) == status


@pytest.mark.parametrize("call", [append, attend])
def test_layouts_that_the_operators_do_not_take(call):
    for dtype, D in (("f16", 64), ("f32", 64), ("fp8", 64), ("bf16", 96), ("fp8_scaled", 32), ("bf16", 512)):
        assert call(ctx(dtype, D, H=4)) == T.TL_ELAYOUT, (dtype, D)


@pytest.mark.parametrize("kw", [
    dict(k=rows(None)), dict(v=rows(FAKE + 8)), dict(k=rows(row=132)), dict(v=rows(head=65)),
    dict(heads=4), dict(heads=4, q=rows()), dict(heads=4, q_out=rows()), dict(q=rows(), q_out=rows()),
    dict(heads=4, q=rows(row=256), q_out=rows(row=192)),              # results over each other
    dict(heads=4, q=rows(row=256), q_out=rows(row=256, head=32)),
    dict(heads=4, q=rows(row=256), q_out=rows(row=512)),              # in place, at other strides
    dict(heads=(1 << 16) + 1, q=rows(), q_out=rows()),
    dict(r=rope(rot_dim=0)), dict(r=rope(rot_dim=80)), dict(r=rope(rot_dim=24)), dict(r=rope(d_cos_sin=None)),
    dict(r=rope(d_cos_sin=FAKE + 8)), dict(r=rope(n_angles=0)), dict(r=rope(flags=2)), dict(r=rope(n_axes=0)),
    dict(r=rope(n_axes=4)), dict(r=rope(n_axes=2)), dict(r=rope(n_axes=2, d_pos=FAKE)),
    dict(r=rope(d_pos=FAKE + 2)), dict(r=rope(pair_axis=ctypes.cast(AXIS, ctypes.c_void_p))),
])
def test_append_refusals(kw):
    assert append(ctx(), **kw) == T.TL_EINVAL


@pytest.mark.parametrize("kw,status", [
    (dict(heads=0), T.TL_EINVAL), (dict(heads=3), T.TL_EINVAL), (dict(heads=1 << 17), T.TL_EINVAL),
    (dict(flags=2), T.TL_EINVAL), (dict(scale=float("nan")), T.TL_EINVAL), (dict(scale=float("inf")), T.TL_EINVAL),
    (dict(q=rows(None)), T.TL_EINVAL), (dict(out=rows(row=128)), T.TL_EINVAL), (dict(out=rows(row=0)), T.TL_EINVAL),
    (dict(out=rows(row=-256)), T.TL_EINVAL), (dict(lse=FAKE + 1), T.TL_EINVAL),
    (dict(ws=None), T.TL_EINVAL), (dict(ws=FAKE + 4), T.TL_EINVAL), (dict(ws_bytes=64), T.TL_ERANGE),
])
def test_attend_refusals(kw, status):
    assert attend(ctx(), **kw) == status


def test_null_arguments():
    lib, c = T.lib(), ctx()
    b, r, p = ctypes.byref(batch()), ctypes.byref(rows()), ctypes.byref(cache(c))
    assert lib.tl_append(None, None, 0, b, None, r, r, 0, None, None, p, None) == T.TL_EINVAL
    assert lib.tl_append(c.handle, None, 0, None, None, r, r, 0, None, None, p, None) == T.TL_EINVAL
    assert lib.tl_append(c.handle, None, 0, b, None, None, r, 0, None, None, p, None) == T.TL_EINVAL
    assert lib.tl_append(c.handle, None, 0, b, None, r, r, 0, None, None, None, None) == T.TL_EINVAL
    assert lib.tl_attend(None, None, 0, b, 2, r, p, 1.0, 0, r, None, FAKE, 1 << 40) == T.TL_EINVAL
    assert lib.tl_attend(c.handle, None, 0, b, 2, None, p, 1.0, 0, r, None, FAKE, 1 << 40) == T.TL_EINVAL
    assert lib.tl_attend(c.handle, None, 0, b, 2, r, None, 1.0, 0, r, None, FAKE, 1 << 40) == T.TL_EINVAL
    assert lib.tl_attend(c.handle, None, 0, b, 2, r, p, 1.0, 0, None, None, FAKE, 1 << 40) == T.TL_EINVAL
    assert lib.tl_attend_workspace_bytes(None, 4, 1, 1) == 0
    assert T.tl_attend_workspace_bytes(c, 3, 1, 1) == 0


def test_nothing_to_do():
    for b in (batch(n_rows=0), batch(n_reqs=0, d_row_off=None, d_kv_len=None, d_tables=None)):
        assert append(ctx(), b=b) == T.TL_OK
        assert attend(ctx(), b=b) == T.TL_OK


def test_binding_refuses_tensors_that_do_not_fit():
    c = ctx()
    x = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device memory"):
        T.tl_append(c, None, 0, batch(), cache(c), x, x)
    with pytest.raises(ValueError, match="bf16"):
        T.tl_append(c, None, 0, batch(), cache(c), x.float(), x)
    with pytest.raises(ValueError, match="heads"):
        T.tl_append(c, None, 0, batch(), cache(c), x[:, :1], x)
    with pytest.raises(ValueError, match="one shape"):
        T.tl_append(c, None, 0, batch(), cache(c), x, x, None, x)
    with pytest.raises(ValueError, match="shape"):
        T.tl_attend(c, None, 0, batch(), cache(c), x, x[:1], FAKE, 64)
    with pytest.raises(ValueError, match="device memory"):
        T.make_batch(1, 2, torch.zeros(2, dtype=torch.int32), FAKE, FAKE, 4)
    with pytest.raises(ValueError, match="axes"):
        T.make_rope(torch.zeros(8, 32, 2, device="meta"), 64, None, [0] * 5)


@pytest.mark.parametrize("L,H,D,P,ppb", [(4, 4, 64, 16, 1), (32, 8, 128, 16, 1), (3, 1, 64, 104, 2), (2, 6, 256, 32, 1),
                                          (1, 1, 1, 1, 1), (2, 1000, 1, 1, 1), (2, 8, 128, 128, 1)])
def test_scaled_layouts_match_the_oracle(L, H, D, P, ppb):
    lay = ref.Layout(L, H, D, 5, P, (), (), ppb)
    c = T.tl_ctx_create(b"tenant", b"model", L, H, D, "fp8_scaled", P, pages_per_block=ppb)
    assert (c.slab_bytes, c.record_bytes, c.payload_offset) == (lay.slab_bytes, lay.record_bytes, lay.payload_offset)
    assert c.slab_bytes % 1024 == 0 and 0 <= c.slab_bytes - (P * H * D + H) < 1024
    assert (c.chunks_per_slab, c.n_segments) == (lay.chunks_per_slab, lay.n_segments)
    assert T.tl_ns_digest(c) == ref.namespace_digest(b"tenant", b"model", lay)


def test_number_formats_of_the_oracle():
    """The oracle's e4m3 against torch's, whose rounding is to nearest even too."""
    r = np.random.default_rng(0)
    x = np.concatenate([r.standard_normal(20000) * 2.0 ** r.integers(-12, 7, 20000), pc._E4M3[:127],
                        (pc._E4M3[:126] + pc._E4M3[1:127]) / 2, [0.0, -0.0, np.inf, np.nan]]).astype(np.float32)
    x = np.clip(x, -448, 448)
    x[-2:] = np.inf, np.nan
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    got = pc.e4m3_codes(x)
    nan = want & 127 == 127
    assert np.array_equal(nan, got & 127 == 127) and np.array_equal(got[~nan], want[~nan])
    back = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.nan_to_num(back, nan=9e9), np.nan_to_num(pc.e4m3_values(np.arange(256)), nan=9e9))
    for a, b in ((448.0, 127), (448.1, 128), (1.75 * 2 ** -109, 10), (2.0 ** -140, 10), (0.0, 10), (3.3e38, 247)):
        assert pc.scale_byte(a) == b
