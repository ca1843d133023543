"""Small batches on a paged cache for the operator tests, and the operators in
plain host arithmetic: appended bytes exactly (32-bit rotation, every operation
rounded; e4m3 and bf16 rounding to nearest even), attention in 64 bits."""
import math

import numpy as np
import torch

from paper_2609_39358_amd import taliesin as T
from paper_2609_39358_amd.device import PagedCache

DEV = "cuda"


def page_bytes(P, H, D, cache):
    n = P * H * D * (2 if cache == "bf16" else 1)
    return n if cache == "bf16" else -(-(n + H) // 1024) * 1024


class Paged:
    """One layer's cache of `kv_len` tokens per request on the host: codes as
    values [n][H][D] (64 bits) and as page bytes, in random pages of a pool whose
    other bytes would spoil any result (NaN)."""

    def __init__(self, seed, P, H, D, cache, q_len, kv_len, window=0, pad=0, layers=1, layer=0, group_of=None):
        self.r = np.random.default_rng(seed)
        self.P, self.H, self.D, self.cache = P, H, D, cache
        self.q_len, self.kv_len, self.window = list(q_len), list(kv_len), window
        self.n, self.rows = len(q_len), sum(q_len)
        self.layers, self.layer = layers, layer
        self.width = max(1, max(-(-k // P) for k in kv_len))
        used = sum(-(-k // P) for k in kv_len)
        self.n_pages = used + 3
        ids = self.r.permutation(self.n_pages)[:used].astype(np.int32)
        self.table = np.full((self.n, self.width), -1, np.int32)
        at = 0
        for i, k in enumerate(kv_len):
            m = -(-k // P)
            self.table[i, :m] = ids[at:at + m]
            at += m
        self.stride = page_bytes(P, H, D, cache) + pad
        self.code_bytes = P * H * D * (2 if cache == "bf16" else 1)
        self.pages = [np.full((self.n_pages, self.stride), 0xFF, np.uint8) for _ in range(2)]  # K, V
        groups = 1 if group_of is None else max(group_of) + 1
        self.group = 0 if group_of is None else group_of[layer]
        self.n_groups = groups
        windows = [0] * layers
        windows[layer] = window
        self.ctx = T.tl_ctx_create(b"tenant", b"model", layers, H, D, cache, P, windows, group_of)
        assert self.ctx.slab_bytes == page_bytes(P, H, D, cache)

    def codes(self, kv):
        """[pages][P][H][D] view of the page bytes: u8 codes or bf16 bits."""
        x = self.pages[kv]
        if self.cache == "bf16":
            x = x.view(np.uint16)
        n, size = self.H * self.D, x.itemsize
        return np.lib.stride_tricks.as_strided(x, (self.n_pages, self.P, self.H, self.D),
                                               (x.strides[0], n * size, self.D * size, size))

    def scales(self, kv):
        return self.pages[kv][:, self.code_bytes:self.code_bytes + self.H]

    def fill(self, amp=1.0, spread=0):
        """Values in every token's place up to kv_len: N(0, 1) times amp, and page
        scales `spread` powers of two apart. Rows past kv_len stay NaN."""
        for kv in range(2):
            for i, k in enumerate(self.kv_len):
                for j in range(-(-k // self.P)):
                    p, m = self.table[i, j], min(self.P, k - j * self.P)
                    x = self.r.standard_normal((m, self.H, self.D)).astype(np.float32) * amp
                    if self.cache == "bf16":
                        self.codes(kv)[p, :m] = bf16_bits(x)
                    else:
                        e = self.r.integers(-spread, spread + 1, self.H) if spread else np.zeros(self.H, int)
                        self.codes(kv)[p, :m] = e4m3_codes(x * 32)
                        self.scales(kv)[p] = (127 - 5 + e).astype(np.uint8)
        return self

    def values(self, kv, i):
        """Request i's tokens as values [kv_len][H][D], 64 bits; a page that the
        table does not name gives NaN."""
        out = np.full((self.kv_len[i], self.H, self.D), np.nan)
        for j in range(-(-self.kv_len[i] // self.P)):
            p, m = self.table[i, j], min(self.P, self.kv_len[i] - j * self.P)
            if not 0 <= p < self.n_pages:
                continue
            x = self.codes(kv)[p, :m]
            if self.cache == "bf16":
                out[j * self.P:j * self.P + m] = bf16_values(x)
            else:
                out[j * self.P:j * self.P + m] = e4m3_values(x) * np.exp2(self.scales(kv)[p].astype(float) - 127)[None, :, None]
        return out

    # ---- on the device
    def up(self):
        self.dk, self.dv = (torch.from_numpy(p.copy()).to(DEV) for p in self.pages)
        other = torch.zeros((self.n_pages, self.stride), dtype=torch.uint8, device=DEV)
        ks, vs = [other] * self.layers, [other] * self.layers
        ks[self.layer], vs[self.layer] = self.dk, self.dv
        self.paged = PagedCache(self.layers, self.n_pages, self.stride, DEV, ks, vs)
        self.row_off = np.concatenate([[0], np.cumsum(self.q_len)]).astype(np.int32)
        tables = np.full((self.n_groups, self.n, self.width), -1, np.int32)
        tables[self.group] = self.table
        self.d = [torch.from_numpy(x).to(DEV) for x in (self.row_off, np.array(self.kv_len, np.int64).astype(np.uint32).view(np.int32), tables)]
        return self

    def batch(self, rows=None):
        return T.make_batch(self.n, self.rows if rows is None else rows, *self.d, self.width)


# ---- number formats -----------------------------------------------------------
def bf16_bits(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)


def bf16_values(bits):
    return (np.ascontiguousarray(bits).astype(np.uint32) << 16).view(np.float32).astype(float)


_E4M3 = np.array([(-1) ** (c >> 7) * ((1 + (c & 7) / 8) * 2.0 ** ((c >> 3 & 15) - 7) if c >> 3 & 15 else (c & 7) / 8 * 2.0 ** -6)
                  if c & 127 != 127 else np.nan for c in range(256)])


def e4m3_values(codes):
    return _E4M3[codes]


def e4m3_codes(x):
    """Nearest code, ties to the even one; what is not finite: NaN. |x| <= 448."""
    x = np.asarray(x, float)
    pos = _E4M3[:127]
    with np.errstate(invalid="ignore"):
        y = np.where(np.isfinite(x), np.abs(x), 0.0)
        hi = np.clip(np.searchsorted(pos, y), 1, 126)
        lo = hi - 1
        up, down = pos[hi] - y, y - pos[lo]
        code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
        code = np.where(y == 0, 0, code)
    code = np.where(np.isfinite(x), code, 127)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_byte(amax):
    b = 10
    while amax > 448 * 2.0 ** (b - 127):
        b += 1
    return b


# ---- the operators ---------------------------------------------------------------
def rotate(x, cs, pos, axis, rot, adjacent):
    """x [T][h][D] f32 by cs [angles][rot / 2][2]; pos [axes][T]."""
    x = np.array(x, np.float32)
    for p in range(rot // 2):
        a, b = (2 * p, 2 * p + 1) if adjacent else (p, p + rot // 2)
        at = pos[axis[p]]
        c, s = cs[at, p, 0][:, None], cs[at, p, 1][:, None]
        u, w = x[:, :, a].copy(), x[:, :, b].copy()
        with np.errstate(all="ignore"):
            x[:, :, a] = u * c - w * s
            x[:, :, b] = w * c + u * s
    return x


def append(c: Paged, k, v):
    """Writes rotated keys and values [rows][H][D] f32 into c.pages."""
    at = 0
    for i in range(c.n):
        for first, end in _fragments(c, i):
            page, o = c.table[i, first // c.P], first % c.P
            rows = slice(at + first - (c.kv_len[i] - c.q_len[i]), at + end - (c.kv_len[i] - c.q_len[i]))
            for kv, x in ((0, k[rows]), (1, v[rows])):
                if c.cache == "bf16":
                    c.codes(kv)[page, o:o + end - first] = bf16_bits(x)
                    continue
                for h in range(c.H):
                    y = np.abs(x[:, h])
                    y = y[np.isfinite(y)]
                    b = scale_byte(float(y.max()) if y.size else 0.0)
                    if o:
                        old = int(c.scales(kv)[page, h])
                        if b > old:
                            held = e4m3_values(c.codes(kv)[page, :o, h]) * 2.0 ** (old - b)
                            c.codes(kv)[page, :o, h] = e4m3_codes(held)
                        b = max(b, old)
                    c.scales(kv)[page, h] = b
                    c.codes(kv)[page, o:o + end - first, h] = e4m3_codes(x[:, h].astype(float) * 2.0 ** (127 - b))
        at += c.q_len[i]


def _fragments(c, i):
    pos = c.kv_len[i] - c.q_len[i]
    while pos < c.kv_len[i]:
        end = min(c.kv_len[i], pos // c.P * c.P + c.P)
        yield pos, end
        pos = end


def attend(c: Paged, q, scale, all_keys=False):
    """(out, lse, bound of out's error, bound of lse's error) for q [rows][Hq][D]
    in 64 bits. The bounds follow from what is rounded: the weights and the
    result to bf16, scores and sums in 32 bits. bf16 has 8 significant bits: half
    a unit in the last place is up to 2^-8 of the value (1 + 2^-8 rounds to 1)."""
    rows, Hq, D = q.shape
    G = Hq // c.H
    out, lse = np.zeros((rows, Hq, D)), np.full((rows, Hq), -np.inf)
    tol, ltol = np.zeros((rows, Hq, D)), np.zeros((rows, Hq))
    at = 0
    for i in range(c.n):
        k, v = c.values(0, i), c.values(1, i)
        named = np.repeat((c.table[i] >= 0) & (c.table[i] < c.n_pages), c.P)[:c.kv_len[i]]
        for t in range(c.q_len[i]):
            pos = c.kv_len[i] - c.q_len[i] + t
            j = np.arange(c.kv_len[i])
            seen = named.copy()
            if not all_keys:
                seen &= j <= pos
                if c.window:
                    seen &= j > pos - c.window
            if not seen.any():
                continue
            for h in range(Hq):
                kk, vv = k[seen, h // G], v[seen, h // G]
                x = q[at + t, h]
                s = kk @ x * scale
                size = (np.abs(kk) @ np.abs(x)).max() * abs(scale)
                ds = size * 2.0 ** -19 + 2.0 ** -20 * (np.abs(s).max() + 16)  # sums of D products; the exponent's rounding
                w = np.exp(s - s.max())
                out[at + t, h] = w @ vv / w.sum()
                lse[at + t, h] = s.max() + math.log(w.sum())
                tol[at + t, h] = (w @ np.abs(vv) / w.sum()) * (2 * 2.0 ** -8 * 1.01 + 2 * ds) + 1e-30
                ltol[at + t, h] = 2 * ds + 1e-5
        at += c.q_len[i]
    return out, lse, tol, ltol
