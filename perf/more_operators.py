"""Performance cases of what an engine does with drafted tokens and with branches of a
request on a paged KV cache: new tokens appended with their queries and keys normed per
head (`tl_append` with a norm), a tree of drafted tokens attending to the cache
(`tl_attend` with a tree), the rows that were accepted moved together (`tl_keep`), and the
pages of branches: shared, copied, taken and freed (`tl_pages_*`).

A case is a dict of plain values:
  kind       norm        norm and rotate q and k, write k and v into one layer's pages
             tree        every query sees the request's tokens before the tree, and those
                         new ones that its mask names
             keep        some of the requests' new tokens stay and move together, all layers
             fork        the last step's branches are freed; new ones share their parents'
                         full pages, get a copy of the last one, and room for more tokens
             copy        pages, or the first rows of them, to other pages, all layers
  heads, q_heads, dim, page_tokens, layers   the cache's geometry (norm, tree: one layer)
  pad        bytes between one page's end and the next page's start
  cache      "bf16", or "fp8_scaled": 8-bit codes (e4m3) and a power-of-two scale for each
             page and head, behind the page's codes
  window     > 0: a query sees only the last `window` tokens before its own position
  requests, median, longest, sigma   how many tokens the requests hold before the call
             (lognormal, cut to [longest / 32, longest])
  new        new tokens of a request; `ragged`: they have 1 to `new` (by turns)
  branch     tree: a node's parent is one of so many nodes before it; norm: > 0, the new
             tokens are such a tree and have its positions
  center     norm: the mean is taken off first; per_head: weights of each head's own
  rot        norm: rotated elements of a head; adjacent: a pair is elements 2i, 2i + 1
  keep       keep: new tokens that stay, at most; keep_first: so many of them are the first
             ones, which stay where they are; the others lie behind the middle
  beams      fork: branches of each request before the step (they share its pages)
  children   fork: new branches in all, of branches at random
  room       fork: tokens that each new branch gets room for
  pages      copy: pages that are copied; whole: every row of them

Scaled 8-bit caches: a page of P tokens holds P * heads * dim codes and then one byte per
head, b, for the scale 2^(b - 127). Writing rows of a page keeps one scale for all its rows:
the larger of the page's own and the smallest power of two, not below 2^-117, that brings the
new rows' largest finite value to at most 448; rows before them are rounded again if it rose.
Writing a page's first row starts it afresh. Values that are not finite become NaN."""
import math
import random
import statistics

import torch

own = False  # False: the operators in elementary torch operations; True: the library's kernels

DEV = "cuda"
EPS = 1e-6  # of the norms
TINY = dict(heads=4, q_heads=8, dim=64, page_tokens=16, layers=1, pad=0, window=0)
MID = dict(TINY, heads=8, q_heads=32, dim=128)  # an 8B-class model with grouped K/V heads
CORPUS = dict(TINY, heads=16, q_heads=32, dim=128)  # the 31B-class model of the paper's corpus
HYBRID = dict(CORPUS, page_tokens=256, window=1024)  # a sliding-window layer of the hybrid model
WIDE = dict(TINY, heads=6, q_heads=24, dim=256, page_tokens=32, pad=1024)
ODD_PAGES = dict(TINY, heads=1, q_heads=8, dim=64, page_tokens=104)  # pages of 104 tokens, one K/V head

NORM = dict(kind="norm", sigma=1.0, ragged=False, branch=0, center=False, per_head=False, adjacent=False)
TREE = dict(kind="tree", sigma=1.0, ragged=False)
KEEP = dict(kind="keep", sigma=1.0, ragged=False, keep_first=1)
FORK = dict(kind="fork", sigma=0.5)
COPY = dict(kind="copy")


def listed():
    return [
        # one decode step of a few short chats on a small model: launches and latency
        dict(TINY, **NORM, name="norm_decode_tiny", cache="fp8_scaled", rot=64, requests=4, median=700, longest=1024, new=1),
        # the drafted trees of a serving batch on an 8B-class model, at their positions
        dict(MID, **dict(NORM, branch=8, ragged=True), name="norm_draft_batch", cache="fp8_scaled", rot=128, requests=96, median=4096, longest=32768, new=24),
        # a long prefill chunk of the 31B-class model on bf16 pages, norms with means and each head's weights
        dict(CORPUS, **dict(NORM, center=True, per_head=True), name="norm_prefill", cache="bf16", rot=64, requests=3, median=5000, longest=9001, new=8191),
        # eight drafted tokens of one short chat: latency
        dict(TINY, **TREE, name="tree_tiny", cache="fp8_scaled", branch=4, requests=1, median=1024, longest=1024, new=8),
        # a serving batch whose requests drafted up to 32 tokens each, some of them none
        dict(MID, **dict(TREE, ragged=True), name="tree_batch", cache="fp8_scaled", branch=12, requests=48, median=4096, longest=32768, new=32),
        # 64 drafted tokens behind the restored 97,000-token corpus
        dict(CORPUS, **TREE, name="tree_corpus", cache="fp8_scaled", branch=12, requests=1, median=96999, longest=96999, new=64),
        # trees of more nodes than a mask's word has bits on a sliding-window layer in bf16
        dict(HYBRID, **dict(TREE, sigma=0.2), name="tree_window", cache="bf16", branch=20, requests=12, median=20000, longest=30001, new=77),
        # a serving batch's accepted drafts, all layers of an 8B-class model
        dict(MID, **dict(KEEP, ragged=True), name="keep_drafts", layers=32, cache="fp8_scaled", requests=96, median=500, longest=1000, new=48, keep=7),
        # one long request cut down to its first tokens and its last ones, on bf16 pages
        dict(CORPUS, **dict(KEEP, keep_first=4), name="keep_recent", layers=12, cache="bf16", requests=1, median=37, longest=37, new=20011, keep=8003),
        # four branches of one short chat go on as four of two of them: latency
        dict(TINY, **FORK, name="fork_tiny", layers=4, cache="fp8_scaled", requests=1, median=301, longest=301, beams=4, children=4, room=1),
        # a serving batch with branches: 256 new ones of 256, all layers of an 8B-class model
        dict(MID, **FORK, name="fork_batch", layers=32, cache="fp8_scaled", requests=32, median=400, longest=1500, beams=8, children=256, room=20),
        # pages that an engine moves itself, partly filled ones
        dict(CORPUS, **COPY, name="copy_pages", layers=12, cache="bf16", pages=301, whole=False),
    ]


LARGEST = {"bytes": 1.5e9, "flops": 1.0e12}  # of a drawn case
PLAIN = 12e9  # bytes of a drawn case's scores, and of its gathered keys, in 32 bits
HELD = 3e9  # bytes of a drawn case's cache


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        case = dict(rng.choice((TINY, MID, MID, CORPUS, CORPUS, HYBRID, WIDE, ODD_PAGES)))
        what = rng.choice(("norm", "norm", "tree", "tree", "tree", "keep", "keep", "fork", "fork", "copy"))
        case["cache"] = rng.choice(("fp8_scaled", "fp8_scaled", "bf16"))
        longest = size(64, 65536)
        case.update(requests=size(1, 192), longest=longest, median=max(1, int(longest * rng.uniform(0.1, 1.0))))
        if what == "norm":
            case.update(NORM, center=rng.random() < 0.3, per_head=rng.random() < 0.3, adjacent=rng.random() < 0.3,
                        rot=rng.choice((case["dim"], case["dim"], case["dim"] // 2)), new=rng.choice((1, size(2, 64), size(2, 8192))))
            if 1 < case["new"] <= 64:
                case.update(branch=size(1, 20), ragged=rng.random() < 0.5)
        elif what == "tree":
            case.update(TREE, branch=size(1, 24), new=size(2, 160), ragged=rng.random() < 0.5)
        elif what == "keep":
            case.update(KEEP, layers=size(1, 48), new=size(4, 160), median=min(case["median"], 2000), longest=min(longest, 2000))
            if rng.random() < 0.3:
                case.update(requests=size(1, 4), new=size(500, 20000))
            case.update(ragged=rng.random() < 0.5 and case["new"] <= 160, keep=rng.randint(1, max(1, case["new"] * 2 // 5)), keep_first=rng.randint(0, 4))
        elif what == "fork":
            case.update(FORK, layers=size(1, 48), requests=size(1, 64), beams=size(1, 16), children=size(1, 512), room=size(1, 64),
                        median=min(case["median"], 2000), longest=min(longest, 2000))
        else:
            case.update(COPY, layers=size(1, 48), pages=size(1, 1000), whole=rng.random() < 0.5)
        w = work(case)
        scores = keys = 0
        if what == "tree":
            new, held = _lengths(case)
            scores = len(new) * max(new) * max(held) * case["q_heads"] * 4
            keys = len(new) * max(held) * case["heads"] * case["dim"] * 4
        if w["bytes"] <= LARGEST["bytes"] and w["flops"] <= LARGEST["flops"] and max(scores, keys) <= PLAIN and _cache_pages(case) * _stride(case) * 2 * case["layers"] <= HELD:
            return case


# ---- sizes -------------------------------------------------------------------
def _held(c):
    """Tokens that every request holds before the call."""
    n, held = c["requests"], []
    for i in range(n):
        z = statistics.NormalDist().inv_cdf((i + 0.5) / n) * c["sigma"]
        held.append(int(min(max(c["median"] * math.exp(z), c["longest"] / 32, 1), c["longest"])))
    return held


def _lengths(c):
    """New tokens of every request, and the tokens that its cache holds after them."""
    held = _held(c)
    new = [c["new"] if not c["ragged"] else 1 + (c["new"] - 1) * (i * 7 % 10) // 9 for i in range(len(held))]
    return new, [a + b for a, b in zip(new, held)]


def _kept(c, new):
    """How many of a request's new tokens stay, and how many of those do not move."""
    n = min(c["keep"], max(1, new * 2 // 5))
    return n, min(c["keep_first"], n)


def _code_bytes(c):
    return c["page_tokens"] * c["heads"] * c["dim"] * (1 if c["cache"] == "fp8_scaled" else 2)


def _page_bytes(c):
    """One page of one layer's K (or V): whole KiB, the scales behind the codes."""
    held = _code_bytes(c) + (c["heads"] if c["cache"] == "fp8_scaled" else 0)
    return -(-held // 1024) * 1024


def _stride(c):
    return _page_bytes(c) + c["pad"]


def _spans(c):
    """The pages of each request that a call touches: an append and a keep those from the first
    new row on, a window layer those in its window."""
    P, spans = c["page_tokens"], []
    for a, b in zip(*_lengths(c)):
        first = 0
        if c["kind"] in ("norm", "keep"):
            first = (b - a) // P
        elif c["window"]:
            first = max(0, b - a + 1 - c["window"]) // P
        spans.append((first, -(-b // P)))
    return spans


def _grown(c):
    """fork: tokens of each branch of a request behind those that its branches share."""
    return [1 + (7 * i) % 61 for i in range(c["requests"])]


def _cache_pages(c):
    if c["kind"] == "copy":
        return 2 * c["pages"] + c["pages"] // 4
    P = c["page_tokens"]
    if c["kind"] == "fork":
        prompts = [-(-h // P) for h in _held(c)]
        own_pages = [-(-(h + g) // P) - h // P for h, g in zip(_held(c), _grown(c))]
        each = 2 + -(-c["room"] // P)
        used = sum(prompts) + c["beams"] * sum(own_pages) + c["children"] * each
    else:
        used = sum(b - a for a, b in _spans(c))
    return used + used // 8 + 1


def work(case):
    c, row = case, case["heads"] * case["dim"] * (1 if case["cache"] == "fp8_scaled" else 2)
    query = c["q_heads"] * c["dim"] * 2
    if c["kind"] == "copy":
        rows = c["pages"] * (c["page_tokens"] if c["whole"] else (c["page_tokens"] + 1) / 2)
        return {"bytes": rows * row * 4 * c["layers"] + 12 * c["pages"], "flops": 0}
    if c["kind"] == "fork":
        part = [(h + g) % c["page_tokens"] for h, g in zip(_held(c), _grown(c))]
        width = max(-(-(h + g + c["room"]) // c["page_tokens"]) for h, g in zip(_held(c), _grown(c)))
        rows = c["children"] * sum(part) / len(part)
        return {"bytes": rows * row * 4 * c["layers"] + 12 * width * c["children"] + 8 * _cache_pages(c), "flops": 0}
    new, held = _lengths(c)
    if c["kind"] == "norm":
        # q and k and v read, q written, k and v written, the rows of the angle table
        per = 2 * query + 2 * (2 * c["heads"] * c["dim"]) + 2 * row + 4 * c["rot"]
        return {"bytes": sum(new) * per, "flops": sum(new) * (c["q_heads"] + c["heads"]) * (c["rot"] * 3 + c["dim"] * 4)}
    if c["kind"] == "keep":
        moved = sum(n - m for n, m in (_kept(c, a) for a in new))
        return {"bytes": moved * row * 4 * c["layers"] + 8 * sum(_kept(c, a)[0] for a in new), "flops": 0}
    pairs = read = 0
    for a, b in zip(new, held):
        w = c["window"] or b
        pairs += a * (min(b - a, w) + 1)  # itself among the new tokens, at least
        read += min(b, w + a - 1)
    return {"bytes": read * 2 * row + sum(new) * (2 * query + 4 * c["q_heads"] + 8 * -(-c["new"] // 64)), "flops": 4 * c["dim"] * c["q_heads"] * pairs}


# ---- inputs ------------------------------------------------------------------
def _scale_byte(amax):
    """b of the smallest 2^(b - 127), from 2^-117 on, with amax <= 448 * 2^(b - 127)."""
    mantissa, exponent = torch.frexp(amax)  # amax = mantissa * 2^exponent, mantissa in [0.5, 1)
    e = exponent - 9 + (mantissa > 0.875).to(exponent.dtype)  # 448 = 0.875 * 2^9
    return torch.where(amax > 0, (e + 127).clamp(min=10), 10).to(torch.uint8)


def _two_to(b):
    return (b.to(torch.int32) << 23).view(torch.float32)  # b is 10 or more


def _fill(c, buf, g):
    """Pages of values as layers leave them: N(0, 1) times a level of each head."""
    n, (P, H, D) = buf.shape[0], (c["page_tokens"], c["heads"], c["dim"])
    buf.zero_()
    level = torch.rand((H, 1), generator=g, device=DEV) * 1.5 + 0.5
    step = max(1, (1 << 28) // (P * H * D))
    for a in range(0, n, step):
        m = min(step, n - a)
        x = torch.randn((m, P, H, D), generator=g, device=DEV).mul_(level)
        codes = buf[a:a + m, :_code_bytes(c)]
        if c["cache"] == "bf16":
            codes.view(torch.bfloat16).copy_(x.reshape(m, -1))
            continue
        b = _scale_byte(x.abs().amax((1, 3)))
        codes.view(torch.float8_e4m3fn).copy_((x / _two_to(b)[:, None, :, None]).to(torch.float8_e4m3fn).reshape(m, -1))
        buf[a:a + m, _code_bytes(c):_code_bytes(c) + H] = b


def _trees(c, new, rng):
    """Nodes' parents: one of the `branch` nodes before; the first node has none."""
    return [[-1] + [rng.randint(max(0, i - c["branch"]), i - 1) for i in range(1, a)] for a in new]


def _seen(trees, words):
    """A mask for each node: itself and its ancestors; and its depth."""
    masks, depths = [], []
    for parents in trees:
        m, d = [], []
        for i, p in enumerate(parents):
            m.append((m[p] if i else 0) | 1 << i)
            d.append(d[p] + 1 if i else 0)
        masks += m
        depths += d
    low = [[(m >> 64 * w) & (2 ** 64 - 1) for w in range(words)] for m in masks]
    return torch.tensor([[x - 2 ** 64 if x >> 63 else x for x in r] for r in low], dtype=torch.int64), depths


def _inputs(c, seed):
    """What both forms take, from the seed alone."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rng = random.Random(seed)
    P, H, D = c["page_tokens"], c["heads"], c["dim"]
    n_pages = _cache_pages(c)
    buf = torch.empty((2 * c["layers"], n_pages, _stride(c)), dtype=torch.uint8, device=DEV)  # layer l: K 2l, V 2l + 1
    for x in buf:
        _fill(c, x, g)
    s = {"case": c, "buf": buf}

    def on(x, dtype=torch.int32):
        return torch.tensor(x, dtype=dtype).to(DEV)

    ids = list(range(n_pages))
    rng.shuffle(ids)
    if c["kind"] == "copy":
        n = c["pages"]
        s.update(src=on(ids[:n]).view(1, n), dst=on(ids[n:2 * n]).view(1, n), rows=on([P if c["whole"] else rng.randint(1, P) for _ in range(n)]))
        return s
    if c["kind"] == "fork":
        width = max(-(-(h + a + c["room"]) // P) for h, a in zip(_held(c), _grown(c)))
        refs, tables, lens = [0] * n_pages, [], []
        for h, a in zip(_held(c), _grown(c)):
            shared = [ids.pop() for _ in range(h // P)]
            for _ in range(c["beams"]):
                mine = shared + [ids.pop() for _ in range(-(-(h + a) // P) - h // P)]
                for p in mine:
                    refs[p] += 1
                tables.append(mine + [-1] * (width - len(mine)))
                lens.append(h + a)
        n = c["children"]
        s.update(width=width, refs=on(refs).view(1, -1), tables=on(tables).view(1, len(lens), width), kv_len=on(lens), branches=len(lens),
                 parent=on([rng.randrange(len(lens)) for _ in range(n)]), out_tables=torch.full((1, n, width), -1, dtype=torch.int32, device=DEV),
                 out_len=torch.zeros(n, dtype=torch.int32, device=DEV), want=torch.zeros(n, dtype=torch.int32, device=DEV))
        return s
    new, held = _lengths(c)
    n, T = len(new), sum(new)
    width = max(-(-k // P) for k in held)
    tables = [[-1] * width for _ in range(n)]
    for r, (a, b) in enumerate(_spans(c)):
        tables[r][a:b] = [ids.pop() for _ in range(a, b)]
    off = [0]
    for a in new:
        off.append(off[-1] + a)
    s.update(tokens=T, requests=n, width=width, tables=on(tables).view(1, n, width), row_off=on(off), kv_len=on(held), max_new=max(new), max_held=max(held))
    if c["kind"] == "keep":
        keep, count = [0] * T, []
        for r, a in enumerate(new):
            k, first = _kept(c, a)
            if c["new"] > 1000:  # the last ones
                rest = range(a - (k - first), a)
            else:  # nodes of a draft's deeper levels
                rest = sorted(rng.sample(range(max(first, a - a // 2), a), min(k - first, a // 2)))
            kept = list(range(first)) + list(rest)
            keep[off[r]:off[r] + len(kept)] = kept
            count.append(len(kept))
        s.update(keep=on(keep), n_keep=on(count))
        return s
    if c["kind"] == "tree" or c["branch"]:
        seen, depths = _seen(_trees(c, new, rng), -(-max(new) // 64))
        s["seen"] = seen.to(DEV)
        s["pos"] = on([b - a + d for a, b, o in zip(new, held, off) for d in depths[o:o + a]])
    if c["kind"] == "tree":
        s["q"] = torch.randn((T, c["q_heads"], D), generator=g, device=DEV).mul_(1.5).to(torch.bfloat16)
        return s
    # queries, keys and values as the slices of one projection's output
    Hq = c["q_heads"]
    qkv = torch.randn((T, Hq + 2 * H, D), generator=g, device=DEV)
    qkv.mul_(torch.rand((1, Hq + 2 * H, 1), generator=g, device=DEV) * 3 + 0.25).add_(torch.randn((1, Hq + 2 * H, 1), generator=g, device=DEV) * 0.25)
    s["qkv"] = qkv = qkv.to(torch.bfloat16)
    s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    for name, heads in (("q_weight", Hq), ("k_weight", H)):
        s[name] = 1 + 0.2 * torch.randn((heads, D) if c["per_head"] else (D,), generator=g, device=DEV)
    half, rows = c["rot"] // 2, max(held)
    freq = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
    angle = torch.arange(rows, dtype=torch.float64, device=DEV)[:, None] * freq
    s["cos_sin"] = torch.stack((angle.cos(), angle.sin()), -1).float()
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    from paper_2609_39358_amd import taliesin as T
    from paper_2609_39358_amd.device import PagedCache

    c, L = case, case["layers"]
    s["T"] = T
    s["ctx"] = T.tl_ctx_create(b"perf-tenant", b"perf-model", L, c["heads"], c["dim"], c["cache"], c["page_tokens"], [c["window"]] * L)
    n_pages, stride = s["buf"].shape[1:]
    s["paged"] = PagedCache(L, n_pages, stride, DEV, [s["buf"][2 * l] for l in range(L)], [s["buf"][2 * l + 1] for l in range(L)])
    s["cache"] = s["paged"].tl()
    if c["kind"] == "copy":
        return s
    if c["kind"] == "fork":
        s["pool"] = T.make_pool(s["refs"])
        s["ws_bytes"] = T.tl_pages_workspace_bytes(s["ctx"], c["children"], n_pages)
        s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device=DEV)
        s["status"] = torch.empty(c["children"], dtype=torch.uint8, device=DEV)
        s["took"] = torch.empty(c["children"], dtype=torch.uint8, device=DEV)
        return s
    s["batch"] = T.make_batch(s["requests"], s["tokens"], s["row_off"], s["kv_len"], s["tables"], s["width"])
    if c["kind"] == "keep":
        s["len_out"] = torch.empty(s["requests"], dtype=torch.int32, device=DEV)
        s["status"] = torch.empty(s["requests"], dtype=torch.uint8, device=DEV)
        return s
    s["out"] = torch.empty((s["tokens"], c["q_heads"], c["dim"]), dtype=torch.bfloat16, device=DEV)
    if c["kind"] == "norm":
        s["rope"] = T.make_rope(s["cos_sin"], c["rot"], s.get("pos"), adjacent=c["adjacent"])
        s["norm"] = T.make_norm(s["q_weight"], s["k_weight"], EPS, center=c["center"])
        return s
    s["tree"] = T.make_tree(s["seen"], s["pos"])
    s["lse"] = torch.empty((s["tokens"], c["q_heads"]), dtype=torch.float32, device=DEV)
    s["ws_bytes"] = T.tl_attend_workspace_bytes(s["ctx"], c["q_heads"], s["requests"], s["tokens"])
    s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device=DEV)
    return s


# ---- one pass ------------------------------------------------------------------
def _pages_out(s):
    """The cache's pages as values: bf16, or the codes and the scales."""
    c, n, buf = s["case"], _code_bytes(s["case"]), s["buf"]
    if c["cache"] == "bf16":
        return [buf[:, :, :n].view(torch.bfloat16)]
    return [buf[:, :, :n].view(torch.float8_e4m3fn), buf[:, :, n:n + c["heads"]].view(torch.float8_e8m0fnu)]


def run(s):
    if not own:
        return {"norm": _plain_norm, "tree": _plain_tree, "keep": _plain_keep, "fork": _plain_fork, "copy": _plain_copy}[s["case"]["kind"]](s)
    T, c, stream = s["T"], s["case"], torch.cuda.current_stream()
    if c["kind"] == "norm":
        T.tl_append(s["ctx"], stream, 0, s["batch"], s["cache"], s["k"], s["v"], rope=s["rope"], q=s["q"], q_out=s["out"], norm=s["norm"])
        return {"q": s["out"], "pages": _pages_out(s)}
    if c["kind"] == "tree":
        T.tl_attend(s["ctx"], stream, 0, s["batch"], s["cache"], s["q"], s["out"], s["ws"], s["ws_bytes"], lse=s["lse"], tree=s["tree"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["kind"] == "keep":
        T.tl_keep(s["ctx"], stream, s["batch"], s["cache"], s["n_keep"], s["keep"], s["len_out"], s["status"])
        return {"pages": _pages_out(s), "kv_len": s["len_out"], "status": s["status"]}
    if c["kind"] == "copy":
        T.tl_pages_copy(s["ctx"], stream, s["cache"], c["pages"], s["src"], s["dst"], s["rows"])
        return {"pages": _pages_out(s)}
    n, width = c["children"], s["width"]
    T.tl_pages_free(s["ctx"], stream, s["pool"], n, s["out_tables"], width)
    T.tl_pages_fork(s["ctx"], stream, s["pool"], s["cache"], s["branches"], s["kv_len"], s["tables"], n, s["parent"], s["out_len"], s["out_tables"],
                    width, s["ws"], s["ws_bytes"], s["status"])
    torch.add(s["out_len"], c["room"], out=s["want"])
    T.tl_pages_take(s["ctx"], stream, s["pool"], n, s["out_len"], s["want"], s["out_tables"], width, s["ws"], s["ws_bytes"], s["took"])
    return {"pages": _pages_out(s), "tables": s["out_tables"], "kv_len": s["out_len"], "refs": s["refs"], "status": s["status"], "took": s["took"]}


def _places(s):
    """(request, index among its new tokens, position) of every new token."""
    t = torch.arange(s["tokens"], device=DEV)
    off = s["row_off"].long()
    r = torch.searchsorted(off[1:], t, right=True)
    return r, t - off[r], s["kv_len"].long()[r] - (off[r + 1] - t)


def _normed(s, x, weight):
    x = x.float()
    if s["case"]["center"]:
        x = x - x.mean(-1, keepdim=True)
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight


def _rotate(s, x, position):
    c, half = s["case"], s["case"]["rot"] // 2
    cs = s["cos_sin"][s["pos"].long() if "pos" in s else position]
    cos, sin = cs[..., 0][:, None], cs[..., 1][:, None]
    turned, rest = x[..., :c["rot"]], x[..., c["rot"]:]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if c["adjacent"] else (turned[..., :half], turned[..., half:])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).flatten(-2) if c["adjacent"] else torch.cat((a, b), -1)
    return torch.cat((turned, rest), -1)


def _plain_norm(s):
    P = s["case"]["page_tokens"]
    r, _, position = _places(s)
    page, row = s["tables"][0].long()[r, position // P], position % P
    k = _rotate(s, _normed(s, s["k"], s["k_weight"]), position)
    q = _rotate(s, _normed(s, s["q"], s["q_weight"]), position).to(torch.bfloat16)
    return {"q": q, "pages": _put(s, torch.stack((k, s["v"].float())), page, row)}


def _put(s, x, page, row):
    """x [slabs, rows, heads, dim] into the rows (page, row), no two of which are one place."""
    c, (S, n) = s["case"], s["buf"].shape[:2]
    P, H, D = shape = (c["page_tokens"], c["heads"], c["dim"])
    out = _pages_out(s)
    if c["cache"] == "bf16":
        out[0].unflatten(2, shape)[:, page, row] = x.to(torch.bfloat16)
        return out
    codes, scales = out[0].unflatten(2, shape), s["buf"][:, :, _code_bytes(c):_code_bytes(c) + H]
    largest = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)  # [S, rows, H]
    largest = torch.zeros((S, n, H), device=DEV).scatter_reduce_(1, page[None, :, None].expand(S, -1, H), largest, "amax")
    first = torch.full((n,), P, device=DEV).scatter_reduce_(0, page, row, "amin")  # first row that is written; P: none
    held = torch.where((first == 0)[:, None], 0, scales)
    b = torch.where((first < P)[:, None], torch.maximum(_scale_byte(largest), held), scales)
    rose = ((b != scales) & (first < P)[:, None]).any(0).any(-1) & (first > 0)  # pages whose earlier rows are rounded again
    at = rose.nonzero()[:, 0]
    again = (torch.arange(P, device=DEV) < first[at, None])[..., None, None]
    rounded = (codes[:, at].float() * (_two_to(scales[:, at]) / _two_to(b[:, at]))[:, :, None, :, None]).to(torch.float8_e4m3fn)
    codes.view(torch.uint8)[:, at] = torch.where(again, rounded.view(torch.uint8), codes.view(torch.uint8)[:, at])
    scales.copy_(b)
    x = x / _two_to(b)[:, page][..., None]
    x = torch.where(x.isfinite(), x, float("nan"))
    codes.view(torch.uint8)[:, page, row] = x.to(torch.float8_e4m3fn).view(torch.uint8)
    return out


def _plain_tree(s):
    c, buf = s["case"], s["buf"]
    P, H, D, G, n = c["page_tokens"], c["heads"], c["dim"], c["q_heads"] // c["heads"], s["requests"]
    j = torch.arange(s["max_held"], device=DEV)
    i = torch.arange(s["max_new"], device=DEV)
    held, off = s["kv_len"].long(), s["row_off"].long()
    before = held - (off[1:] - off[:-1])
    page = s["tables"][0].long()[:, j // P]
    there = (j < held[:, None]) & (page >= 0)
    page = page.clamp(min=0)
    pages = _pages_out(s)

    def rows(kv):
        x = pages[0][kv].unflatten(1, (P, H, D))
        if c["cache"] == "bf16":
            x = x[page, j % P].float()
        else:
            x = x.view(torch.uint8)[page, j % P].view(torch.float8_e4m3fn).float()
            x = x * _two_to(buf[kv, :, _code_bytes(c):_code_bytes(c) + H])[page][..., None]
        return torch.where(there[..., None, None], x, 0.0).transpose(1, 2).contiguous()  # [n, H, held, D]

    k, v = rows(0), rows(1)
    t = (off[:-1, None] + i).clamp(max=s["tokens"] - 1)  # [n, new]
    q = s["q"].float()[t].unflatten(2, (H, G)).permute(0, 2, 3, 1, 4).reshape(n, H, G * s["max_new"], D)
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(D)).unflatten(2, (G, s["max_new"]))
    bits = ((s["seen"][..., None] >> torch.arange(64, device=DEV)) & 1).flatten(1).bool()[t]  # [n, new, 64 * words]
    rel = j - before[:, None]
    named = bits.gather(2, rel.clamp(0, bits.shape[2] - 1)[:, None].expand(-1, s["max_new"], -1))
    early = (rel < 0)[:, None].expand(-1, s["max_new"], -1)
    if c["window"]:
        early = early & (j > (s["pos"].long()[t] - c["window"])[..., None])
    seen = there[:, None] & (early | ((rel >= 0)[:, None] & named))
    scores.masked_fill_(~seen[:, None, None], float("-inf"))
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top.isfinite(), top, 0.0)
    weights = scores.sub_(top).exp_()
    total = weights.sum(-1, keepdim=True)
    out = torch.matmul(weights.flatten(2, 3), v).unflatten(2, (G, s["max_new"]))
    out = torch.where(total > 0, out / total, 0.0)
    lse = (top + total.log()).squeeze(-1)
    r, at, _ = _places(s)
    out = out.permute(0, 3, 1, 2, 4).flatten(2, 3)[r, at]
    return {"out": out.to(torch.bfloat16), "lse": lse.permute(0, 3, 1, 2).flatten(2, 3)[r, at]}


def _plain_keep(s):
    c, P, H, D = s["case"], s["case"]["page_tokens"], s["case"]["heads"], s["case"]["dim"]
    r, i, position = _places(s)
    before = position - i
    at = before + s["keep"].long()
    moved = (i < s["n_keep"].long()[r]) & (at != position)
    table = s["tables"][0].long()
    r, position, at = r[moved], position[moved], at[moved]
    pages = _pages_out(s)
    page = table[r, at // P]
    x = pages[0].unflatten(2, (P, H, D)).view(torch.bfloat16 if c["cache"] == "bf16" else torch.uint8)[:, page, at % P]
    if c["cache"] == "bf16":
        x = x.float()
    else:
        x = x.view(torch.float8_e4m3fn).float() * _two_to(s["buf"][:, :, _code_bytes(c):_code_bytes(c) + H])[:, page][..., None]
    out = _put(s, x, table[r, position // P], position % P)
    new = s["row_off"][1:] - s["row_off"][:-1]
    return {"pages": out, "kv_len": s["kv_len"] - new + s["n_keep"], "status": torch.ones_like(s["n_keep"], dtype=torch.uint8)}


def _copy_rows(s, src, dst, rows):
    """The first `rows` rows of pages src (whole numbers; and their scales) to pages dst."""
    c, P = s["case"], s["case"]["page_tokens"]
    row = _code_bytes(c) // P
    take = torch.arange(s["buf"].shape[2], device=DEV)
    n = _code_bytes(c) + (c["heads"] if c["cache"] == "fp8_scaled" else 0)
    mine = torch.where(take < _code_bytes(c), take < (rows * row)[:, None], take < n)
    s["buf"][:, dst] = torch.where(mine, s["buf"][:, src], s["buf"][:, dst])


def _plain_copy(s):
    _copy_rows(s, s["src"][0].long(), s["dst"][0].long(), s["rows"].long())
    return {"pages": _pages_out(s)}


def _fresh(refs, wanted):
    """The free pages, lowest first, for the places that are wanted, in order."""
    order = torch.argsort((refs > 0).int(), stable=True)
    return order[(wanted.flatten().cumsum(0) - 1).clamp(min=0)].view(wanted.shape)


def _plain_fork(s):
    c, P, refs = s["case"], s["case"]["page_tokens"], s["refs"][0]
    table, out = s["tables"][0].long(), s["out_tables"][0]

    def count(pages, by):
        refs.index_add_(0, pages.clamp(min=0).flatten(), torch.where(pages >= 0, by, 0).flatten().to(torch.int32))

    count(out.long(), -1)
    parent = s["parent"].long()
    kv = s["kv_len"].long()[parent]
    full, part = kv // P, kv % P
    col = torch.arange(s["width"], device=DEV)
    rows = table[parent]
    shared = torch.where(col < full[:, None], rows, -1)
    last = rows.gather(1, full.clamp(max=s["width"] - 1)[:, None])[:, 0]
    wants = (part > 0) & (last >= 0)
    fresh = _fresh(refs, wants)
    mine = torch.where((col == full[:, None]) & wants[:, None], fresh[:, None], shared)
    count(mine, 1)
    _copy_rows(s, torch.where(wants, last, 0), torch.where(wants, fresh, 0), torch.where(wants, part, 0))
    s["out_len"].copy_(kv)
    lacks = (col >= -(-kv // P)[:, None]) & (col < -(-(kv + c["room"]) // P)[:, None])
    took = torch.where(lacks, _fresh(refs, lacks), -1)
    count(took, 1)
    out.copy_(torch.where(lacks, took, mine))
    fine = torch.ones_like(parent, dtype=torch.uint8)
    return {"pages": _pages_out(s), "tables": s["out_tables"], "kv_len": s["out_len"], "refs": s["refs"], "status": fine, "took": fine.clone()}


# ---- the definition in 64 bits ---------------------------------------------------
def exact(case, seed):
    """Request by request, from the definition. Codes are given before they are rounded."""
    s = _inputs(case, seed)
    return {"norm": _exact_norm, "tree": _exact_tree, "keep": _exact_keep, "fork": _exact_fork, "copy": _exact_copy}[case["kind"]](s)


class _Store:
    """Pages in 64 bits: values [slabs][pages][P][H][D] (scaled: codes) and powers of two [slabs][pages][H]."""

    def __init__(self, s):
        c = s["case"]
        P, H, D, n, f64 = c["page_tokens"], c["heads"], c["dim"], _code_bytes(c), torch.float64
        self.scaled = c["cache"] == "fp8_scaled"
        x = s["buf"][:, :, :n].view(torch.float8_e4m3fn if self.scaled else torch.bfloat16)
        self.x = x.to(f64).unflatten(2, (P, H, D))
        self.power = s["buf"][:, :, n:n + H].to(f64) - 127 if self.scaled else None

    def write(self, P, table, start, x):
        """x [slabs, rows, H, D] to the positions from `start` on of one request."""
        end = start + x.shape[1]
        for at in range(start // P * P, end, P):
            p, a, b = table[at // P], max(at, start), min(at + P, end)
            part = x[:, a - start:b - start]
            if not self.scaled:
                self.x[:, p, a - at:b - at] = part
                continue
            need = torch.ceil(torch.log2(part.abs().amax((1, 3)).clamp(min=1e-300) / 448)).clamp(min=-117)
            e = torch.maximum(need, self.power[:, p]) if a > at else need
            if a > at:
                self.x[:, p, :a - at] *= torch.exp2(self.power[:, p] - e)[:, None, :, None]
            self.x[:, p, a - at:b - at] = part / torch.exp2(e)[:, None, :, None]
            self.power[:, p] = e

    def read(self, P, table, positions):
        """[slabs, rows, H, D] of one request."""
        at = torch.tensor(positions, device=DEV)
        page = torch.tensor(table, device=DEV)[at // P]
        x = self.x[:, page, at % P]
        return x * torch.exp2(self.power[:, page])[..., None] if self.scaled else x

    def out(self):
        x = self.x.flatten(2)
        return [x, torch.exp2(self.power)] if self.scaled else [x]


def _exact_norm(s):
    c, f64 = s["case"], torch.float64
    half, off, held = c["rot"] // 2, s["row_off"].tolist(), s["kv_len"].tolist()
    store = _Store(s)
    q = torch.empty(s["q"].shape, dtype=f64, device=DEV)

    def of(x, weight, pos):
        x = x.to(f64)
        if c["center"]:
            x = x - x.sum(-1, keepdim=True) / c["dim"]
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["dim"] + EPS) * weight.to(f64)
        z = x.clone()
        for p in range(half):
            cs = s["cos_sin"][pos, p].to(f64)
            a, b = (2 * p, 2 * p + 1) if c["adjacent"] else (p, p + half)
            z[:, :, a] = x[:, :, a] * cs[:, None, 0] - x[:, :, b] * cs[:, None, 1]
            z[:, :, b] = x[:, :, a] * cs[:, None, 1] + x[:, :, b] * cs[:, None, 0]
        return z

    for r in range(s["requests"]):
        lo, hi = off[r], off[r + 1]
        start = held[r] - (hi - lo)
        pos = s["pos"][lo:hi].long() if "pos" in s else torch.arange(start, held[r], device=DEV)
        q[lo:hi] = of(s["q"][lo:hi], s["q_weight"], pos)
        store.write(c["page_tokens"], s["tables"][0, r].tolist(), start, torch.stack((of(s["k"][lo:hi], s["k_weight"], pos), s["v"][lo:hi].to(f64))))
    return {"q": q, "pages": store.out()}


def _exact_tree(s):
    c, f64 = s["case"], torch.float64
    P, H, D, G, n = c["page_tokens"], c["heads"], c["dim"], c["q_heads"] // c["heads"], _code_bytes(c)
    off, held, seen = s["row_off"].tolist(), s["kv_len"].tolist(), s["seen"].tolist()
    out = torch.zeros((s["tokens"], c["q_heads"], D), dtype=f64, device=DEV)
    lse = torch.full((s["tokens"], c["q_heads"]), float("-inf"), dtype=f64, device=DEV)
    for r in range(s["requests"]):
        lo, hi, last = off[r], off[r + 1], held[r]
        new = hi - lo
        start = last - new
        first = max(0, start - c["window"] + 1) if c["window"] else 0
        j = torch.arange(first, last, device=DEV)
        page = s["tables"][0, r].long()[j // P]
        hidden = torch.zeros((new, last - first), dtype=torch.bool, device=DEV)
        names = torch.tensor([[not seen[lo + t][m // 64] >> m % 64 & 1 for m in range(new)] for t in range(new)], device=DEV)
        hidden[:, start - first:] = names
        if c["window"]:
            hidden[:, :start - first] = j[:start - first] <= s["pos"][lo:hi, None].long() - c["window"]
        for h in range(H):
            both = []
            for kv in range(2):
                codes = s["buf"][kv, :, :n].view(torch.uint8 if c["cache"] != "bf16" else torch.bfloat16).unflatten(1, (P, H, D))[page, j % P, h]
                x = codes.to(f64) if c["cache"] == "bf16" else codes.view(torch.float8_e4m3fn).to(f64) * torch.exp2(s["buf"][kv, page, n + h].to(f64) - 127)[:, None]
                both.append(x)
            for g in range(h * G, h * G + G):
                z = (s["q"][lo:hi, g].to(f64) @ both[0].T / math.sqrt(D)).masked_fill(hidden, float("-inf"))
                lse[lo:hi, g] = torch.logsumexp(z, -1)
                out[lo:hi, g] = torch.softmax(z, -1) @ both[1]
    return {"out": out, "lse": lse}


def _exact_keep(s):
    P, off, held = s["case"]["page_tokens"], s["row_off"].tolist(), s["kv_len"].tolist()
    store, keep, count, length = _Store(s), s["keep"].tolist(), s["n_keep"].tolist(), []
    for r in range(s["requests"]):
        table, kept = s["tables"][0, r].tolist(), keep[off[r]:off[r] + count[r]]
        start = held[r] - (off[r + 1] - off[r])
        length.append(start + len(kept))
        stay = 0
        while stay < len(kept) and kept[stay] == stay:
            stay += 1
        if stay < len(kept):
            store.write(P, table, start + stay, store.read(P, table, [start + k for k in kept[stay:]]))
    return {"pages": store.out(), "kv_len": torch.tensor(length), "status": torch.ones(len(length), dtype=torch.uint8)}


def _exact_copy(s):
    store = _Store(s)
    for a, b, rows in zip(s["src"][0].tolist(), s["dst"][0].tolist(), s["rows"].tolist()):
        store.x[:, b, :rows] = store.x[:, a, :rows]
        if store.scaled:
            store.power[:, b] = store.power[:, a]
    return {"pages": store.out()}


def _exact_fork(s):
    c, P, store = s["case"], s["case"]["page_tokens"], _Store(s)
    refs, tables, lens = s["refs"][0].tolist(), s["tables"][0].tolist(), s["kv_len"].tolist()
    out, length = [], []

    def lowest():
        lowest.at = next(i for i in range(lowest.at, len(refs)) if refs[i] <= 0)
        refs[lowest.at] = 1
        return lowest.at

    lowest.at = 0
    for p in s["parent"].tolist():
        kv = lens[p]
        row = [x if i < kv // P else -1 for i, x in enumerate(tables[p])]
        for x in row:
            if x >= 0:
                refs[x] += 1
        if kv % P and tables[p][kv // P] >= 0:
            a, b = tables[p][kv // P], lowest()
            row[kv // P] = b
            store.x[:, b, :kv % P] = store.x[:, a, :kv % P]
            if store.scaled:
                store.power[:, b] = store.power[:, a]
        out.append(row)
        length.append(kv)
    for row, kv in zip(out, length):
        for i in range(-(-kv // P), -(-(kv + c["room"]) // P)):
            row[i] = lowest()
    fine = torch.ones(len(out), dtype=torch.uint8)
    return {"pages": store.out(), "tables": torch.tensor([out]), "kv_len": torch.tensor(length), "refs": torch.tensor([refs]), "status": fine, "took": fine.clone()}
