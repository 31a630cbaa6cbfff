"""Attention over a 4-bit cache with block ids outside the pool: the tokens of such a block are skipped, in both kinds of attention and in
every form of them; the rest of the request counts as if they did not exist."""
import numpy as np
import pytest
import torch

import paper_2601_11822_amd as rs
from tests import kv4_ref as R
from tests.gpu_util import to_bits
from tests.test_gpu_kv4 import Cache, i32, wide

pytestmark = pytest.mark.gpu


def reported(c, side):
    with pytest.raises(rs.RapidServeError) as e:
        c.c.sync(side)
    assert e.value.code == rs.RS_ERR_BAD_BLOCK
    c.c.sync(side)   # once


def held_over_what_is_left(c, got, q, tab, r, first, name):
    """got, q [rows, ...] of request r at positions first ..: attention over the tokens whose block is one of the pool."""
    n = first + got.shape[0]
    there = np.array([0 <= tab[r, t // 16] < c.n_blocks for t in range(n)])
    ids = np.where((tab[r] >= 0) & (tab[r] < c.n_blocks), tab[r], 0)
    k, v = R.gather(c.ref[0], c.hd, ids, n)
    rows = range(got.shape[0]) if got.shape[0] <= 70 else sorted({i for i in (0, 1, 15, 16, 31, 32, 47, 48, 63, 64, 100, 500, 2023, 2040) if i < got.shape[0]} | {got.shape[0] - 1})
    worst = 0.0
    for i in rows:
        keep = there[:first + i + 1]
        want, bound = R.attention(R.f64(q[i:i + 1]), k[:first + i + 1][keep], v[:first + i + 1][keep], int(keep.sum()) - 1)
        if not keep.any():
            assert (got[i] == 0).all(), (name, i)
            continue
        fine = bool(np.isfinite(got[i]).all())
        assert fine, (name, i)
        worst = max(worst, float(np.max(np.abs(got[i] - want[0]) / np.maximum(bound[0], 1e-30))))
    print(f"  {name}: {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0, name


@pytest.mark.parametrize("heads,lens,starts,bad", [
    ((8, 2, 128), [100, 40], [30, 0], [[1, 5, 6], [0, 2]]),          # keys whole; a request whose first rows see nothing
    ((4, 4, 64), [100, 40], [30, 0], [[1, 5, 6], [0, 2]]),
    ((8, 2, 128), [19], [3000], [[0, 3, 4, 77, 188]]),               # keys in pieces
    ((4, 4, 64), [2], [700], [[0, 1, 2, 3, 20, 43]]),                # a key tile of which nothing is left
    ((8, 2, 128), [5], [40], [[0, 1, 2]]),                           # nothing left at all
    ((128, 8, 128), [2041], [0], [[0, 7, 30, 31, 32, 33, 126]]),     # workgroups of eight waves
], ids=lambda x: str(x)[:18])
def test_prompts_skip_a_block_that_is_none(heads, lens, starts, bad):
    held = [s + n for s, n in zip(starts, lens)]
    c = Cache(heads, sum(-(-n // 16) for n in held) + 4, max_prefill=sum(lens), seed=11)
    tab, _ = c.tables(held)
    c.fill(tab, held)
    for r, which in enumerate(bad):
        tab[r, which] = [c.n_blocks + 3 if i % 2 else -2 for i in range(len(which))]
    dtab = torch.from_numpy(tab).cuda()
    cu, W = np.concatenate([[0], np.cumsum(lens)]), c.Hq * c.hd
    q = c.queries(int(cu[-1]))
    dq, out = wide(q, W, W), torch.full((int(cu[-1]), W), 7.0, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    c.c.kv4_prefill_attention(0, dq, W, out, W, cu, starts, dtab, tab.shape[1])
    reported(c, 0)
    got = R.f64(to_bits(out)).reshape(-1, c.Hq, c.hd)
    for r in range(len(lens)):
        held_over_what_is_left(c, got[cu[r]:cu[r + 1]], q[cu[r]:cu[r + 1]], tab, r, starts[r], f"request {r}")
    c.c.destroy()


@pytest.mark.parametrize("heads,ctx,max_ctx,bad", [
    ((8, 2, 128), [700, 20], 701, [[0, 3, 4, 43], [0, 1]]),                     # whole rows, eight waves
    ((4, 4, 64), [700, 20], 701, [[0, 3, 4, 43], [0, 1]]),
    ((4, 4, 128), [300] + [15] * 79, 301, [[0, 7, 18]] + [[0]] * 79),           # four
    ((4, 4, 64), [300] + [15] * 79, 301, [[0, 7, 18]] + [[0]] * 79),
    ((8, 2, 128), [5000, 40], 9000, [[0, 16, 17, 18, 19, 20, 21, 22, 23, 312], [2]]),   # equal shares
    ((4, 4, 64), [5000, 40], 9000, [[0, 16, 17, 18, 19, 20, 21, 22, 23, 312], [2]]),
], ids=lambda x: str(x)[:18])
def test_decode_rows_skip_a_block_that_is_none(heads, ctx, max_ctx, bad):
    held = [n + 1 for n in ctx]
    c = Cache(heads, sum(-(-n // 16) for n in held) + 4, max_batch=len(ctx), max_context=9000, seed=12)
    tab, _ = c.tables(held)
    c.fill(tab, held)
    for r, which in enumerate(bad):
        tab[r, which] = [c.n_blocks + 3 if i % 2 else -2 for i in range(len(which))]
    tab = np.concatenate([tab, np.full((len(ctx), -(-max_ctx // 16)), -1, np.int32)], 1)
    dtab, dctx, W = torch.from_numpy(tab).cuda(), i32(ctx), c.Hq * c.hd
    q = c.queries(len(ctx))
    dq, out = wide(q, W, W), torch.full((len(ctx), W), 7.0, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    c.c.kv4_decode_attention(0, dq, W, out, W, dctx, dtab, tab.shape[1], len(ctx), max_ctx)
    reported(c, 1)
    got = R.f64(to_bits(out)).reshape(-1, c.Hq, c.hd)
    for r in range(min(len(ctx), 5)):
        held_over_what_is_left(c, got[r:r + 1], q[r:r + 1], tab, r, ctx[r], f"row {r}")
    c.c.destroy()
