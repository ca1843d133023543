"""Branches that draft trees on scaled pages that they share, in every layer: the queries and keys
that a step norms, turns and writes, and what its rows answer, against 64 bits over the
values that the branch's own table names when the tree is attended; before and after the
accepted rows are moved together and branched again."""
import numpy as np
import pytest
import torch

from paper_2609_39358_amd import taliesin as T
from paper_2609_39358_amd.device import PagedCache
from paper_2609_39358_amd.pipeline import NewTokens, PagePool
from tests.test_gpu_branches import D, H, HQ, L, P, PAGES, WIDTH, WORDS, DEV, Model, held, up
from tests.test_gpu_norm import exact
from tests.test_gpu_tree import drafted, words_of

pytestmark = pytest.mark.gpu

EPS = 1e-5


def answers(q, k, v, seen):
    """One row's heads over the keys that it sees, and the bounds of test_gpu_tree: weights and
    results rounded to bf16, half a step of 2^-8 each, scores off by ds."""
    out, tol = np.zeros((HQ, D)), np.zeros((HQ, D))
    for h in range(HQ):
        kk, vv = k[seen, h * H // HQ], v[seen, h * H // HQ]
        s = kk @ q[h] * D ** -0.5
        ds = (np.abs(kk) @ np.abs(q[h])).max() * D ** -0.5 * 2.0 ** -19 + 2.0 ** -20 * (np.abs(s).max() + 16)
        w = np.exp(s - s.max())
        out[h] = w @ vv / w.sum()
        tol[h] = w @ np.abs(vv) / w.sum() * (2 * 2.0 ** -8 * 1.01 + 2 * ds) + 1e-30
    return out, tol


@pytest.mark.parametrize("groups", [None, [0, 1, 0]])
@pytest.mark.parametrize("own_stream", [False, True])
def test_what_the_rows_answer(groups, own_stream):
    ctx = T.tl_ctx_create(b"tenant", b"model", L, H, D, "fp8_scaled", P, [0] * L, groups)
    G, r = ctx.n_groups, np.random.default_rng(7)
    stream = torch.cuda.Stream() if own_stream else None
    model = Model(8, groups)
    cache = PagedCache(L, PAGES, ctx.slab_bytes, DEV)
    for x in cache.k + cache.v:
        x.fill_(0xFF)  # NaN wherever nothing was written
    pool = PagePool(ctx, cache, used=[3], stream=stream)
    cs = model.cos_sin.cpu().numpy()

    def step_of(tables, lens, new, trees, ids):
        """A step through the layers, checked; trees: (masks, depths) of each request."""
        off, before = np.concatenate([[0], np.cumsum(new)]), lens - new
        pos = np.concatenate([b + d for b, (_, d) in zip(before, trees)])
        step = NewTokens(ctx, cache, HQ, sum(new), up(off), up(lens), tables, model.cos_sin, stream,
                         up(np.concatenate([words_of(s, WORDS) for s, _ in trees]).view(np.int64), np.int64), up(pos))
        for l in range(L):
            x = model.table[l, torch.from_numpy(ids).to(DEV)]
            q, k, v = x.split([HQ, H, H], dim=1)
            out = step.layer(l, q, k, v, norm=T.make_norm(*model.weights[l], EPS))
            torch.cuda.synchronize()
            got_q, out, x = step.q.float().cpu().numpy().astype(float), out.float().cpu().numpy(), x.float().cpu().numpy()
            wq, wk = (w.cpu().numpy() for w in model.weights[l])
            want, wide = exact(x[:, :HQ], wq, EPS, False, cs, pos, D)
            assert (np.abs(got_q - want) <= np.abs(want) * 2.0 ** -8 + 1.01 * wide).all()
            keys, wide = exact(x[:, HQ:HQ + H], wk, EPS, False, cs, pos, D)
            host = tables.cpu().numpy()[groups[l] if groups else 0]
            for i, n in enumerate(lens):
                kv = held(ctx, cache, "fp8_scaled", host[i], n)
                pages = cache.k[l].cpu().numpy()[host[i, np.arange(before[i], n) // P]]
                unit = np.exp2(pages[:, P * H * D:P * H * D + H].astype(float) - 127)[:, :, None]
                rows = slice(off[i], off[i + 1])  # rounded to e4m3 once
                bound = np.maximum(np.abs(keys[rows]) * 2.0 ** -4, unit * 2.0 ** -10) + 1.05 * wide[rows]
                assert (np.abs(kv[2 * l, before[i]:] - keys[rows]) <= bound).all()
                for t in range(new[i]):
                    seen = np.concatenate([np.ones(before[i], bool), trees[i][0][t]])
                    want, tol = answers(got_q[off[i] + t], kv[2 * l], kv[2 * l + 1], seen)
                    assert (np.abs(out[off[i] + t] - want) <= tol).all(), (l, i, t)
        assert (step.status == T.ACCEPT).all()
        return step, off

    n = 45  # the prompt: a text is a tree in which all rows see those before them
    tables, lens = torch.full((G, 1, WIDTH), -1, dtype=torch.int32, device=DEV), np.array([n])
    pool.take(up([0]), up(lens), tables)
    torch.cuda.synchronize()
    step_of(tables, lens, np.array([n]), [(np.tril(np.ones((n, n), bool)), np.arange(n))], r.integers(0, 512, n))
    for parents in ([0, 0, 0], [2, 0, 2, 1]):
        old = tables
        tables, d_lens = pool.fork(up(lens), old, up(parents))
        pool.free(old)
        new = r.integers(1, 14, len(parents))
        lens = lens[parents] + new
        pool.take(d_lens, up(lens), tables)
        torch.cuda.synchronize()
        assert (pool.status == T.ACCEPT).all() and d_lens.tolist() == (lens - new).tolist()
        trees = [drafted(r, int(m), 4) for m in new]
        step, off = step_of(tables, lens, new, trees, r.integers(0, 512, sum(new)))
        keep, count = np.zeros(sum(new), np.int64), []
        for i, (see, _) in enumerate(trees):
            path = np.flatnonzero(see[new[i] - 1])
            keep[off[i]:off[i] + len(path)] = path
            count.append(len(path))
        d_lens = step.keep(up(count), up(keep))
        pool.free(tables, d_first=d_lens)
        torch.cuda.synchronize()
        lens = lens - new + count
        assert (step.kept == T.ACCEPT).all() and d_lens.tolist() == lens.tolist()
