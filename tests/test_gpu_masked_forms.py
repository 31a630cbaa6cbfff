"""Windowed and tree attention in the forms that only many keys or many requests lead to (tests/host_masked_check.hip holds the forms that these
sizes take): units of 128 columns over short and odd requests, contexts of more than 32K tokens, keys cut in pieces where results are not
finite, partitions, and recorded graphs."""
import math

import numpy as np
import pytest
import torch

from tests import step_ref as R
from tests import test_gpu_trees as T
from tests import test_gpu_windows as W
from tests.step_ref import Step, i32, wide

pytestmark = pytest.mark.gpu


# ---- units of 128 columns over short requests ----
@pytest.mark.parametrize("heads", R.HEADS + [(64, 4, 64)], ids=str)
@pytest.mark.parametrize("draft", [33, 64])
@pytest.mark.parametrize("times", [1, 10])
def test_short_trees_under_a_bound_of_many_tokens(heads, draft, times):
    ctx = [0, 1, 15, 16, 100, 63, 64, 250, 31] * times
    lens = [draft, 0, 1, draft, draft // 2, draft - 1, 17, draft, 0] * times
    c = Step(heads, sum(-(-(a + b) // 16) for a, b in zip(ctx, lens)) + 1, max_batch=9 * times, max_context=9600, seed=20)
    tab = c.tables([a + b for a, b in zip(ctx, lens)], width=600)
    q = c.queries(sum(lens))
    masks = [m for n in lens for m in T.paths(c.g, n)]
    masks[3] = 0
    got = T.tree(c, tab, ctx, lens, masks, q, max_draft=draft, max_ctx=9600)
    T.check(f"{heads} {draft}", c, tab, ctx, lens, masks, q, got, every=5 * times)
    chain = T.tree(c, tab, ctx, lens, None, q, max_draft=draft, max_ctx=9600)
    T.check(f"{heads} {draft} chains", c, tab, ctx, lens, None, q, chain, every=9 * times)
    c.c.destroy()


@pytest.mark.parametrize("heads,lens,starts", [
    ((64, 16, 64), [700, 0, 300, 33, 1, 290], [0, 7, 16, 31, 200, 5]),
    ((32, 2, 128), [1100, 700, 333, 60, 17], [3, 0, 50, 111, 64]),
    ((64, 16, 64), [330, 37, 1, 16], [40, 300, 250, 112]),
], ids=str)
@pytest.mark.parametrize("window,sinks", [(50, 20), (64, 0), (129, 16), (300, 33), (2 ** 31 - 1, 0)])
def test_short_prompts_of_many_rows(heads, lens, starts, window, sinks):
    total = [s + n for s, n in zip(starts, lens)]
    c = Step(heads, sum(-(-n // 16) for n in total) + 1, max_prefill=sum(lens), max_context=1300, seed=21)
    tab = c.tables(total)
    q = c.queries(sum(lens))
    got = W.prefill(c, tab, lens, starts, window, sinks, q)
    W.check_prefill(f"{heads} {window}+{sinks}", c, tab, lens, starts, window, sinks, q, got, some=31)
    c.c.destroy()


@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 0), (1250, 16)])
def test_prompts_of_more_units_than_compute_units_in_two_teams(window, sinks):
    lens, starts = [1300, 100], [0, 20]
    c = Step((32, 8, 128), 100, max_prefill=1400, max_context=2048, seed=30)
    tab = c.tables([1300, 120])
    q = c.queries(1400)
    got = W.prefill(c, tab, lens, starts, window, sinks, q)
    W.check_prefill(f"{window}+{sinks}", c, tab, lens, starts, window, sinks, q, got, some=67)
    assert torch.equal(got, W.prefill(c, tab, lens, starts, window, sinks, q))
    c.c.destroy()


# ---- more than 32K tokens ----
LONG = 41000


class Needles:
    """A cache whose keys are zero but at `at`, where the score of every query is 40 or more: a row's result is the mean of the values of
    those that it sees, and all its other keys together weigh less than 2^16 e^-40."""

    def __init__(self, heads, total, at, **limits):
        Hq, Hkv, hd = heads
        self.c = c = Step(heads, -(-total // 16) + 3, max_context=-(-total // 16) * 16, fill="nan", seed=22, **limits)
        self.at = np.array(sorted(at))
        self.tab = c.tables([total])
        u = torch.from_numpy(np.sign(c.g.standard_normal((Hkv, hd))).astype(np.float32))
        c.k.zero_()
        c.v.copy_(torch.randn(c.v.shape, generator=torch.Generator().manual_seed(23)))
        blk, slot = torch.as_tensor(self.tab[0][self.at // 16]).long(), torch.as_tensor(self.at % 16)
        c.k[0, blk, slot] = ((2.5 if hd == 64 else 2.0) * u).bfloat16()
        c.push()
        self.q = (2.0 * u).repeat_interleave(Hq // Hkv, 0).bfloat16()
        self.values = c.v[0, blk, slot].double()   # [needles, Hkv, hd]

    def check(self, name, got, sees):
        """got [rows, Hq, hd], sees [rows, needles].  The weights are 1 up to what the exponent of 2 loses (40 log2(e) in two roundings of
        2^-24: within 2^-18 of the sum; as a factor of V it is rounded to 1), sums of some tens of values are within 2^-19 of their size, together
        less than 2^-16 of it; the result is rounded to bf16."""
        n = torch.from_numpy(sees).double()
        assert bool((n.sum(1) > 0).all())
        n = n / n.sum(1, keepdim=True)
        flat = self.values.reshape(len(self.at), -1)
        G = self.c.Hq // self.c.Hkv
        up = lambda x: x.view(len(sees), self.c.Hkv, self.c.hd).repeat_interleave(G, 1)
        want, size = up(n @ flat), up(n @ flat.abs())
        R.held(name, got, want, 2.0 ** -8 * want.abs() + 2.0 ** -16 * size + 2.0 ** -30)


def some_needles(ends):
    """About 30 places: random ones, and those beside the 2048th block of a workgroup that begins with the first."""
    g = np.random.default_rng(24)
    return {0, 32751, 32767, 32768, 32783, 32800, *g.integers(1, LONG, 20).tolist(), *ends}


@pytest.mark.parametrize("heads,rows", [((64, 16, 64), 160), ((64, 16, 64), 300), ((64, 16, 64), 600), ((32, 8, 128), 600), ((32, 8, 128), 1200)], ids=str)
@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 0), (35000, 100)])
def test_prompts_behind_more_than_32k_tokens(heads, rows, window, sinks):
    n = Needles(heads, LONG + rows, some_needles([LONG, LONG + 31, LONG + 100, LONG + rows - 1]), max_prefill=rows)
    q = n.q.expand(rows, -1, -1).contiguous()
    got = W.prefill(n.c, n.tab, [rows], [LONG], window, sinks, q)
    pos = LONG + np.arange(rows)[:, None]
    n.check(f"{heads} {rows} {window}+{sinks}", got, (n.at <= pos) & ((n.at > pos - window) | (n.at < sinks)))
    n.c.c.destroy()


@pytest.mark.parametrize("heads,batch", [((64, 16, 64), 1), ((64, 16, 64), 5), ((64, 16, 64), 9), ((32, 8, 128), 10), ((32, 8, 128), 17)], ids=str)
def test_trees_behind_more_than_32k_tokens(heads, batch):
    """(The requests read one sequence.)"""
    n = Needles(heads, LONG + 64, some_needles([LONG, LONG + 5, LONG + 40, LONG + 63]), max_batch=batch)
    lens = [64 - r for r in range(batch)]
    ctx = [LONG - 16 * r for r in range(batch)]
    q = n.q.expand(sum(lens), -1, -1).contiguous()
    got = T.tree(n.c, np.repeat(n.tab, batch, 0), ctx, lens, None, q, max_draft=64, max_ctx=LONG + 64)
    last = np.concatenate([c + np.arange(m) for c, m in zip(ctx, lens)])[:, None]
    n.check(f"{heads} x {batch}", got, n.at <= last)
    n.c.c.destroy()


@pytest.mark.parametrize("heads,batch", [((64, 16, 64), 1), ((32, 8, 128), 40)], ids=str)
@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 0), (35000, 100)])
def test_decode_rows_behind_more_than_32k_tokens(heads, batch, window, sinks):
    n = Needles(heads, LONG + 1, some_needles([LONG]), max_batch=batch)
    ctx = [LONG - 37 * r for r in range(batch)]
    got = W.decode(n.c, np.repeat(n.tab, batch, 0), ctx, window, sinks, n.q.expand(batch, -1, -1).contiguous(), max_ctx=LONG + 1)
    pos = np.array(ctx)[:, None]
    n.check(f"{heads} x {batch} {window}+{sinks}", got, (n.at <= pos) & ((n.at > pos - window) | (n.at < sinks)))
    n.c.c.destroy()


# ---- keys in pieces ----
@pytest.mark.parametrize("poison", [math.nan, math.inf])
def test_a_decode_row_in_pieces_beside_values_that_are_not_finite(poison):
    """The tokens just outside the window and just behind the sinks hold what must not reach the row; a value that it sees shows."""
    c = Step((32, 8, 128), 200, max_batch=1, max_context=4096, seed=25)
    ctx, window, sinks = 3000, 2000, 5
    tab = c.tables([ctx + 1])
    q = c.queries(1)
    for t in (sinks, sinks + 1, 15, ctx - window, ctx - window - 1):
        c.k[0, tab[0, t // 16], t % 16] = poison
        c.v[0, tab[0, t // 16], t % 16] = poison
    c.push()
    got = W.decode(c, tab, [ctx], window, sinks, q)
    W.check_decode(f"{poison}", c, tab, [ctx], window, sinks, q, got)
    c.v[0, tab[0, 2000 // 16], 2000 % 16, 3, 7] = poison
    c.push()
    shown = W.decode(c, tab, [ctx], window, sinks, q)
    assert bool((~torch.isfinite(shown[0, 12:16, 7])).all())
    shown[0, 12:16, 7] = got[0, 12:16, 7]
    c.v[0, tab[0, 2000 // 16], 2000 % 16, 3, 7] = 0.0
    want, bound = W.expect(c, tab, 0, ctx, q[0], window, sinks)
    want[12:16, 7] = got[0, 12:16, 7].double()
    R.held("the other elements", shown[0], want, bound)
    c.c.destroy()


def test_prompt_rows_in_pieces_beside_values_that_are_not_finite():
    lens, starts, window, sinks = [100], [3000], 3000, 5
    c = Step((32, 8, 128), 200, max_prefill=100, max_context=4096, seed=26)
    tab = c.tables([3100])
    q = c.queries(100)
    c.v[0, tab[0, 3040 // 16], 3040 % 16] = math.inf
    c.k[0, tab[0, 3080 // 16], 3080 % 16] = math.nan
    c.v[0, tab[0, 20 // 16], 20 % 16] = math.nan      # seen by rows up to the position 3019
    c.push()
    got = W.prefill(c, tab, lens, starts, window, sinks, q)
    for i in range(100):
        pos = 3000 + i
        if pos - window < 20 or pos >= 3080:
            assert bool(torch.isnan(got[i]).all()), pos
        elif pos >= 3040:
            assert bool((got[i] == math.inf).all()), pos
        elif i % 4 == 0 or pos in (3020, 3039):
            R.held(f"row at {pos}", got[i], *W.expect(c, tab, 0, pos, q[i], window, sinks))
    c.c.destroy()


@pytest.mark.parametrize("poison", [math.nan, math.inf])
def test_trees_in_pieces_beside_values_that_are_not_finite(poison):
    ctx, lens = [3600, 3591], [40, 39]
    c = Step((32, 8, 128), 460, max_batch=2, max_context=4096, seed=27)
    tab = c.tables([a + b for a, b in zip(ctx, lens)])
    q = c.queries(79)
    hidden = {0, 9, 38}
    masks = [m & ~sum(1 << t for t in hidden) | 1 << (1 + i % 8) for i, m in enumerate([m for n in lens for m in T.paths(c.g, n)])]
    masks[50] |= 1 << 9
    for r in range(2):
        for t in hidden:
            at = ctx[r] + t
            c.k[0, tab[r, at // 16], at % 16] = poison
            c.v[0, tab[r, at // 16], at % 16] = poison
    c.push()
    got = T.tree(c, tab, ctx, lens, masks, q)
    for i in range(79):
        r, at = (0, i) if i < 40 else (1, i - 40)
        if i == 50:
            assert not bool(torch.isfinite(got[i]).any())
        elif i % 5 == 0 or i in (49, 51, 39, 78):
            R.held(f"{r} {at}", got[i], *R.attention(q[i], *c.tokens(tab[r], R.tree_keys(ctx[r], lens[r], masks[i]))))
    c.c.destroy()


def ragged(seed):
    c = Step((32, 8, 128), 900, max_batch=6, max_prefill=200, max_context=4096, seed=seed)
    ctx, lens = [100, 3900, 0, 1500, 37, 2800], [33, 33, 12, 1, 0, 30]
    tab = c.tables([a + b for a, b in zip(ctx, lens)])
    q = c.queries(200)
    return c, ctx, lens, tab, q, [m for n in lens for m in T.paths(c.g, n)]


def test_a_partition_gives_the_same_bits():
    c, ctx, lens, tab, q, masks = ragged(28)
    got = []
    for split in ((256, 256), (128, 128), (32, 224), (224, 32)):
        c.c.set_cu_split(*split)
        got.append((T.tree(c, tab, ctx, lens, masks, q[:109], max_draft=64), W.prefill(c, tab[1:2], [200], [3700], 3500, 4, q)))
    T.check("trees", c, tab, ctx, lens, masks, q, got[0][0], every=9)
    W.check_prefill("rows", c, tab[1:2], [200], [3700], 3500, 4, q, got[0][1], some=50)
    for t, p in got[1:]:
        assert torch.equal(t, got[0][0]) and torch.equal(p, got[0][1])
    c.c.destroy()


def test_both_sides_at_once_and_recorded_graphs():
    """Trees on the decode side while prompt rows run on the other, eager and from a graph each, whose requests change between replays; two
    graphs share the decode side's workspace."""
    c, ctx, lens, tab, q, masks = ragged(29)
    Wd = c.Hq * c.hd
    dt, dc, du, dm = torch.from_numpy(tab).cuda(), i32(ctx), i32([0] + np.cumsum(lens).tolist()), T.i64(masks)
    dq = wide(q, Wd)
    outs = [torch.zeros(200, Wd, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    calls = [lambda: c.c.tree_attention(0, dq, Wd, outs[0], Wd, dc, du, dm, dt, tab.shape[1], 6, 109, 64, 3933),
             lambda: c.c.tree_attention(0, dq, Wd, outs[1], Wd, dc, du, None, dt, tab.shape[1], 6, 109, 33, 3933),
             lambda: c.c.window_prefill_attention(0, dq, Wd, outs[2], Wd, [0, 200], [3700], dt[1:2], tab.shape[1], 3500, 4)]
    streams = [torch.cuda.ExternalStream(c.c.get_stream(s)) for s in (0, 1)]
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in calls]
    for g, call, side in zip(graphs, calls, (1, 1, 0)):
        with torch.cuda.graph(g, stream=streams[side]):
            call()
    for rep in range(4):
        dq.copy_(wide(c.queries(200), Wd))
        if rep:
            dc.copy_(i32([ctx[1], ctx[0], 0, 1500 - rep, 37, 2800 - 64 * rep]))
            dt[0].copy_(torch.from_numpy(tab[1])), dt[1].copy_(torch.from_numpy(tab[1]))
        torch.cuda.synchronize()
        for call in calls:
            call()
        c.c.sync(0), c.c.sync(1)
        want = [o.cpu() for o in outs]
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for g, side in zip(graphs, (1, 1, 0)):
            with torch.cuda.stream(streams[side]):
                g.replay()
        c.c.sync(0), c.c.sync(1)
        for w, o in zip(want, outs):
            assert torch.equal(w, o.cpu()) and float(w.abs().sum()) > 0, rep
    del graphs
    c.c.destroy()
