"""Attention of drafted trees over the bf16 cache against its definition in float64."""
import math

import numpy as np
import pytest
import torch

import paper_2601_11822_amd as rs
from tests import step_ref as R
from tests.step_ref import Step, i32, i64, wide

pytestmark = pytest.mark.gpu


def tree(c, tab, ctx, lens, masks, q, max_draft=None, max_ctx=None, max_rows=None, pad=8, cu=None, layer=0):
    W = c.Hq * c.hd
    cu = [0] + [int(x) for x in np.cumsum(lens)] if cu is None else cu
    total = sum(lens)
    out = torch.full((total + 2, W + 16), math.nan, dtype=torch.bfloat16, device="cuda")
    dq, dt, dc, du = wide(q, W + pad), torch.from_numpy(tab).cuda(), i32(ctx), i32(cu)
    dm = i64(masks) if masks is not None else None
    torch.cuda.synchronize()
    c.c.tree_attention(layer, dq, W + pad, out, W + 16, dc, du, dm, dt, tab.shape[1], len(ctx), total if max_rows is None else max_rows,
                       max_draft or max(max(lens), 1), max_ctx or max(c + n for c, n in zip(ctx, lens)))
    c.c.sync(1)
    out = out.cpu()
    assert bool(torch.isnan(out[:, W:]).all()) and bool(torch.isnan(out[total:]).all())
    return out[:total, :W].view(total, c.Hq, c.hd)


def check(name, c, tab, ctx, lens, masks, q, got, every=1):
    at = 0
    for r, n in enumerate(lens):
        rows = [i for i in range(n) if i % every == 0 or i == n - 1]
        want = []
        for i in rows:
            mask = masks[at + i] if masks is not None else (2 << i) - 1
            want.append(R.attention(q[at + i], *c.tokens(tab[r], R.tree_keys(max(ctx[r], 0), n, mask))))
        if rows:
            R.held(f"{name} request {r}", got[[at + i for i in rows]], torch.stack([w for w, _ in want]), torch.stack([b for _, b in want]))
        at += n


def paths(g, n):
    out = []
    for i, p in enumerate(R.random_tree(g, n)):
        out.append((out[p] if p >= 0 else 0) | 1 << i)
    return out


@pytest.mark.parametrize("heads", R.HEADS + [(64, 4, 64)], ids=str)
@pytest.mark.parametrize("max_draft", [1, 2, 7, 16, 33, 64])
def test_trees(heads, max_draft):
    ctx = [0, 1, 15, 16, 100, 63, 64, 250, 31]
    lens = [max_draft, 0, 1, max_draft, max(max_draft // 2, 1), max_draft, 1, max_draft, 0]
    c = Step(heads, sum(-(-(a + b) // 16) for a, b in zip(ctx, lens)) + 1, max_batch=9, max_context=400, seed=1)
    tab = c.tables([a + b for a, b in zip(ctx, lens)])
    q = c.queries(sum(lens))
    masks = [m for n in lens for m in paths(c.g, n)]
    got = tree(c, tab, ctx, lens, masks, q)
    check(f"{heads} {max_draft}", c, tab, ctx, lens, masks, q, got, every=5)
    chain = tree(c, tab, ctx, lens, None, q)
    check(f"{heads} {max_draft} chains", c, tab, ctx, lens, None, q, chain, every=9)
    c.c.destroy()


@pytest.mark.parametrize("heads,batch,ctx,draft", [
    ((8, 2, 128), 1, 4000, 8),       # keys in pieces
    ((4, 4, 64), 2, 3001, 64),
    ((16, 1, 128), 3, 2500, 40),
    ((32, 8, 128), 40, 600, 33),     # more workgroups than compute units
    ((8, 8, 128), 1, 4000, 3),
    ((32, 4, 64), 30, 555, 5),
], ids=str)
def test_trees_behind_long_contexts(heads, batch, ctx, draft):
    ctxs, lens = [ctx - 13 * i for i in range(batch)], [draft - i % 2 for i in range(batch)]
    c = Step(heads, sum(-(-(a + b) // 16) for a, b in zip(ctxs, lens)) + 1, max_batch=batch, max_context=8192, seed=2)
    tab = c.tables([a + b for a, b in zip(ctxs, lens)])
    q = c.queries(sum(lens))
    masks = [m for n in lens for m in paths(c.g, n)]
    got = tree(c, tab, ctxs, lens, masks, q)
    check(f"{heads} x {batch}", c, tab, ctxs, lens, masks, q, got, every=max(draft * batch // 24, 1))
    assert torch.equal(got, tree(c, tab, ctxs, lens, masks, q))
    c.c.destroy()


def test_any_mask_and_rows_that_see_nothing():
    """Masks need not be ancestors: a row may see later tokens, not itself, or nothing at all; bits behind the request's rows count for nothing."""
    ctx, lens = [0, 0, 37], [9, 64, 12]
    c = Step((8, 2, 128), 12, max_batch=3, max_context=128, seed=3)
    tab = c.tables([a + b for a, b in zip(ctx, lens)])
    q = c.queries(sum(lens))
    masks = [int(x) for x in c.g.integers(0, 2 ** 63, sum(lens), dtype=np.uint64) * np.uint64(2) + np.uint64(1)]
    masks[0], masks[3], masks[20], masks[75], masks[5], masks[30] = 0, ((1 << 55) - 1) << 9, 0, 0, R.FULL, R.FULL
    got = tree(c, tab, ctx, lens, masks, q)
    check("any", c, tab, ctx, lens, masks, q, got)
    assert bool((got[[0, 3, 20]] == 0).all())
    c.c.destroy()


@pytest.mark.parametrize("heads,draft", [((8, 2, 128), 5), ((8, 2, 128), 33), ((4, 4, 64), 12), ((9, 3, 128), 5)], ids=str)
@pytest.mark.parametrize("poison", [math.nan, math.inf])
def test_a_token_off_the_path_does_not_reach_a_row(heads, draft, poison):
    """Every drafted token whose index is a multiple of 4 holds NaN or infinities, and so do the places behind the draft; rows that do not see them are
    as if they were not."""
    ctx, lens = [21, 130], [draft, draft]
    c = Step(heads, 20, max_batch=2, max_context=256, seed=4)
    tab = c.tables([a + b for a, b in zip(ctx, lens)])
    q = c.queries(2 * draft)
    clean = sum(1 << i for i in range(draft) if i % 4)
    masks = [(m & clean) if i % 3 else m for i, m in enumerate([m for n in lens for m in paths(c.g, n)])]
    for r in range(2):
        for t in list(range(0, draft, 4)) + list(range(draft, 16 * -(-(ctx[r] + draft) // 16) - ctx[r])):
            at = ctx[r] + t
            c.v[0, tab[r, at // 16], at % 16] = poison
            if t >= draft:
                c.k[0, tab[r, at // 16], at % 16] = poison
    c.push()
    got = tree(c, tab, ctx, lens, masks, q)
    for r in range(2):
        for i in range(draft):
            m = masks[r * draft + i]
            if m & ~clean:
                assert not bool(torch.isfinite(got[r * draft + i]).any())
            else:
                R.held(f"{r} {i}", got[r * draft + i], *R.attention(q[r * draft + i], *c.tokens(tab[r], R.tree_keys(ctx[r], draft, m))))
    c.c.destroy()


def test_counts_that_contradict_their_bounds():
    """Requests whose rows are out of range are left alone, those whose lengths are get zeros; the others are computed."""
    c = Step((8, 2, 128), 40, max_batch=5, max_context=256, seed=5)
    ctx, lens = [20, 30, 40, 50, 60], [3, 5, 3, 3, 3]
    tab = c.tables([a + b for a, b in zip(ctx, lens)])
    q = c.queries(17)

    def reported(code, **kw):
        W = c.Hq * c.hd
        out = torch.full((17, W), math.nan, dtype=torch.bfloat16, device="cuda")
        a = dict(ctx=ctx, cu=[0, 3, 8, 11, 14, 17], max_rows=17, max_draft=5, max_ctx=63, tab=tab)
        a.update(kw)
        dq, dt, dc, du = wide(q, W), torch.from_numpy(a["tab"]).cuda(), i32(a["ctx"]), i32(a["cu"])
        torch.cuda.synchronize()
        c.c.tree_attention(0, dq, W, out, W, dc, du, None, dt, tab.shape[1], 5, a["max_rows"], a["max_draft"], a["max_ctx"])
        if code:
            with pytest.raises(rs.RapidServeError) as e:
                c.c.sync(1)
            assert e.value.code == code
        c.c.sync(1)
        return out.cpu().view(17, c.Hq, c.hd)

    good = reported(0)
    check("good", c, tab, ctx, lens, None, q, good)
    same = lambda got, rows: torch.equal(got[rows], good[rows])
    for name, kw, code, left, zero in [
        ("too many of one request", dict(max_draft=4), rs.RS_ERR_BAD_ARG, [3, 4, 5, 6, 7], []),
        ("rows behind the last", dict(max_rows=16), rs.RS_ERR_BAD_ARG, [14, 15, 16], []),
        ("descending", dict(cu=[0, 3, 8, 7, 7, 7]), rs.RS_ERR_BAD_ARG, list(range(8, 17)), []),
        ("before the first", dict(cu=[-1, 3, 8, 11, 14, 17]), rs.RS_ERR_BAD_ARG, [0, 1, 2], []),
        ("no request", dict(ctx=[20, -1, 40, 50, 60]), rs.RS_ERR_BAD_BLOCK, [], [3, 4, 5, 6, 7]),
        ("too long", dict(max_ctx=62), rs.RS_ERR_BAD_BLOCK, [], [14, 15, 16]),
        ("far too long", dict(ctx=[20, 30, 2 ** 31 - 1, 50, 60]), rs.RS_ERR_BAD_BLOCK, [], [8, 9, 10]),
    ]:
        got = reported(code, **kw)
        assert bool(torch.isnan(got[left]).all()), name
        assert bool((got[zero] == 0).all()), name
        assert same(got, [i for i in range(17) if i not in left + zero]), name
    bad = tab.copy()
    bad[1, 0], bad[3, 3] = c.n_blocks, -5
    got = reported(rs.RS_ERR_BAD_BLOCK, tab=bad)
    for i in range(5):
        keys = np.array([j for j in R.tree_keys(30, 5, (2 << i) - 1) if j >= 16])
        R.held("over what is left", got[3 + i], *R.attention(q[3 + i], *c.tokens(tab[1], keys)))
    assert same(got, [0, 1, 2, 8, 9, 10, 14, 15, 16])
    c.c.destroy()
