"""Attention over a 4-bit cache in the forms that long contexts and full launches take, against the definition in float64, over values that
show which keys counted; scores that run over hundreds of powers of two; the query's last bits.  tests/host_kv4_check.hip holds that
these sizes take the forms they are about."""
import math

import numpy as np
import pytest
import torch

from tests import kv4_marks as M
from tests import kv4_ref as R
from tests.gpu_util import to_bits
from tests.test_gpu_kv4 import Cache, i32, wide

pytestmark = pytest.mark.gpu


class Marked(Cache):
    """A cache of random keys and marked values."""

    def __init__(self, heads, counts, seed, **kw):
        need = sum(-(-n // 16) for n in counts)
        super().__init__(heads, need + 3, seed=seed, **kw)
        self.ref[0] = M.random_keys(self.g, self.n_blocks, self.Hkv, self.hd)
        self.tab, self.dtab = self.tables(counts)
        for r, n in enumerate(counts):
            M.mark(self.ref[0], self.hd, self.tab[r, :-(-n // 16)])
        self.pool.copy_(torch.from_numpy(self.ref))

    def soft_queries(self, n):
        return R.to_bf16_bits((0.4 * self.g.standard_normal((n, self.Hq, self.hd))).astype(np.float32))


def decode(c, q, ctx, dtab, width, max_ctx):
    W, B = c.Hq * c.hd, len(ctx)
    dq, out, dctx = wide(q, W, W), torch.full((B, W), 7.0, dtype=torch.bfloat16, device="cuda"), i32(ctx)
    torch.cuda.synchronize()
    c.c.kv4_decode_attention(0, dq, W, out, W, dctx, dtab, width, B, max_ctx)
    c.c.sync(1)
    return R.f64(to_bits(out)).reshape(B, c.Hq, c.hd)


def prompts(c, q, cu, starts, dtab, width):
    W, T = c.Hq * c.hd, int(cu[-1])
    dq, out = wide(q, W, W), torch.full((T, W), 7.0, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    c.c.kv4_prefill_attention(0, dq, W, out, W, cu, starts, dtab, width)
    c.c.sync(0)
    return R.f64(to_bits(out)).reshape(T, c.Hq, c.hd)


def near(got, q, k, v, pos, name):
    want, bound = R.attention(R.f64(q[None]), k[:pos + 1], v[:pos + 1], pos)
    assert np.isfinite(got).all(), name
    off = M.worst(got, want[0], bound[0])
    print(f"  {name}: {off:.3f} of the bound", flush=True)
    assert off <= 1, name


@pytest.mark.parametrize("heads,ctx,max_ctx,rows", [
    ((8, 2, 128), [30000, -1, 5], 32768, (0, 2)),                      # shares: 29 pieces to join
    ((4, 4, 64), [20000], 20001, (0,)),                                # 19 pieces
    ((16, 4, 128), [4600] + [33] * 69, 4601, (0, 1, 69)),              # whole rows of four waves, block ids asked for a second time
    ((8, 4, 64), [33] * 30 + [4607] + [33] * 39, 4608, (0, 30, 69)),
    ((16, 16, 64), [17000] * 7 + [17100], 17101, (0, 3, 7)),           # shares of more than 32 units, the same there
    ((16, 16, 128), [17000] * 7 + [17100], 17101, (3,)),
    ((8, 4, 64), [int(x) for x in np.linspace(700, 0, 69)] + [-1], 701, (0, 7, 34, 62, 68)),   # short contexts, whole, four waves
    ((8, 4, 128), [int(x) for x in np.linspace(700, 0, 69)] + [-1], 701, (0, 7, 34, 62, 68)),
], ids=lambda x: str(x)[:24])
def test_decode(heads, ctx, max_ctx, rows):
    c = Marked(heads, [n + 1 for n in ctx], seed=len(ctx) + heads[2], max_batch=len(ctx), max_context=32768)
    tab = np.concatenate([c.tab, np.full((len(ctx), max(0, -(-max_ctx // 16) - c.tab.shape[1])), -1, np.int32)], 1)
    dtab = torch.from_numpy(tab).cuda()
    q = c.soft_queries(len(ctx))
    got = decode(c, q, ctx, dtab, tab.shape[1], max_ctx)
    for r, n in enumerate(ctx):
        if n < 0:
            assert (got[r] == 0).all()
        assert np.isfinite(got[r]).all()
    for r in rows:
        k, v = M.held(c.ref[0], c.hd, tab[r], ctx[r] + 1)
        near(got[r], q[r], k, v, ctx[r], f"row {r}, ctx {ctx[r]}")
    c.c.destroy()


@pytest.mark.parametrize("heads,lens,starts,rows", [
    ((32, 8, 128), [19], [6005], [(0, 0), (0, 18)]),                                      # 24 pieces to join
    ((16, 4, 64), [7, 19], [9000, 6005], [(0, 0), (0, 6), (1, 0), (1, 18)]),              # more than 8
    ((32, 8, 128), [2048], [0], [(0, 0), (0, 31), (0, 32), (0, 1000), (0, 1023), (0, 1024), (0, 2015), (0, 2047)]),   # uncut, all at once: folded
    ((9, 3, 128), [2100, 1900], [0, 0], [(0, 0), (0, 42), (0, 2099), (1, 0), (1, 1000), (1, 1899)]),                   # a fold inside a unit's heads
    ((12, 3, 64), [2100, 1900], [0, 0], [(0, 0), (0, 42), (0, 2099), (1, 0), (1, 1000), (1, 1899)]),
    ((128, 8, 128), [2041, 30], [0, 3000], [(0, 0), (0, 16), (0, 1500), (0, 2040), (1, 0), (1, 29)]),                  # workgroups of eight waves
], ids=lambda x: str(x)[:24])
def test_prompts(heads, lens, starts, rows):
    held = [s + n for s, n in zip(starts, lens)]
    c = Marked(heads, held, seed=len(lens) + heads[0], max_prefill=sum(lens))
    cu = np.concatenate([[0], np.cumsum(lens)])
    q = c.soft_queries(int(cu[-1]))
    got = prompts(c, q, cu, starts, c.dtab, c.tab.shape[1])
    assert np.isfinite(got).all()
    for r in range(len(lens)):
        k, v = M.held(c.ref[0], c.hd, c.tab[r], held[r])
        for i in [i for s, i in rows if s == r]:
            near(got[cu[r] + i], q[cu[r] + i], k, v, starts[r] + i, f"request {r}, row {i}")
    c.c.destroy()


class Steep(Cache):
    """The first request's scores run over hundreds of powers of two; the others' hold a few tokens of any kind."""

    def __init__(self, heads, counts, **kw):
        super().__init__(heads, sum(-(-n // 16) for n in counts) + 3, seed=heads[2], **kw)
        self.tab, self.dtab = self.tables(counts)
        for r, n in enumerate(counts):
            M.mark(self.ref[0], self.hd, self.tab[r, :-(-n // 16)])
            k = np.tile(M.steep_keys(self.g, n, self.hd), (1, self.Hkv // 4, 1))
            for t in range(n):
                codes, scales = R.quantise(k[t])
                kc, _, ks, _ = R.places(self.hd, t % 16)
                blk = self.ref[0, self.tab[r, t // 16]]
                blk[:, kc], blk[:, ks] = codes[..., 0::2] | codes[..., 1::2] << 4, scales
        self.pool.copy_(torch.from_numpy(self.ref))

    def ones(self, n):
        return R.to_bf16_bits((1 + 0.02 * self.g.standard_normal((n, self.Hq, self.hd))).astype(np.float32))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n,rows,max_ctx", [(1500, 2, 1501), (1500, 65, 1501), (5000, 2, 9000), (300, 1, 9000)])   # whole rows of eight waves, of four, shares, one share
def test_decode_with_scores_over_hundreds_of_powers_of_two(hd, n, rows, max_ctx):
    ctx = [n] + [20] * (rows - 1)
    c = Steep((8, 4, hd), [x + 1 for x in ctx], max_batch=rows, max_context=9000)
    tab = np.concatenate([c.tab, np.full((rows, 600), -1, np.int32)], 1)
    q = c.ones(rows)
    got = decode(c, q, ctx, torch.from_numpy(tab).cuda(), tab.shape[1], max_ctx)
    for r in range(min(rows, 3)):
        k, v = M.held(c.ref[0], hd, tab[r], ctx[r] + 1)
        near(got[r], q[r], k, v, ctx[r], f"row {r}")
    c.c.destroy()


@pytest.mark.parametrize("heads,lens,starts", [((8, 4, 64), [200], [0]), ((8, 4, 128), [200], [0]), ((8, 4, 64), [5, 3], [5000, 40]), ((8, 4, 128), [5, 3], [5000, 40]),
                                               ((128, 8, 128), [2041], [0])], ids=str)
def test_prompts_with_scores_over_hundreds_of_powers_of_two(heads, lens, starts):
    held = [s + n for s, n in zip(starts, lens)]
    c = Steep(heads, held, max_prefill=sum(lens))
    cu = np.concatenate([[0], np.cumsum(lens)])
    q = c.ones(int(cu[-1]))
    got = prompts(c, q, cu, starts, c.dtab, c.tab.shape[1])
    for r, n in enumerate(lens):
        k, v = M.held(c.ref[0], c.hd, c.tab[r], held[r])
        for i in sorted({0, 1, 31, 64, 100, 1000, 2000, n - 1} & set(range(n))):
            near(got[cu[r] + i], q[cu[r] + i], k, v, starts[r] + i, f"request {r}, row {i}")
    c.c.destroy()


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64)])
def test_the_query_is_taken_to_its_last_term(heads):
    """64 requests of two tokens, whose scores differ by the small part of a query beside a large one; both kinds of attention."""
    c = Cache(heads, 1, max_prefill=64, max_batch=64)
    k, v = np.zeros((2, c.Hkv, c.hd)), np.zeros((2, c.Hkv, c.hd))
    k[1, :, 5] = 6
    v[0, :, 0] = v[1, :, 1] = 6
    for t in range(2):
        R.put(c.ref[0], c.hd, 0, t, k[t], v[t])
    c.pool.copy_(torch.from_numpy(c.ref))
    tab = torch.zeros((64, 1), dtype=torch.int32, device="cuda")
    q = M.fine_queries(c.g, 64, c.Hq, c.hd)
    for got in (decode(c, q, [1] * 64, tab, 1, 2), prompts(c, q, np.arange(65), [1] * 64, tab, 1)):
        off = 0.0
        for r in range(64):
            want, bound = R.attention(R.f64(q[r:r + 1]), k, v, 1)
            off = max(off, M.worst(got[r], want[0], bound[0]))
        print(f"  {off:.3f} of the bound", flush=True)
        assert off <= 1
    c.c.destroy()
