"""Windowed attention with sinks over the bf16 cache, decode rows and prompt rows, against its definition in float64."""
import math

import numpy as np
import pytest
import torch

import paper_2601_11822_amd as rs
from tests import step_ref as R
from tests.step_ref import Step, i32, wide

pytestmark = pytest.mark.gpu


def decode(c, tab, ctx, window, sinks, q, max_ctx=None, pad=8, layer=0):
    W = c.Hq * c.hd
    out = torch.full((len(ctx), W + 16), math.nan, dtype=torch.bfloat16, device="cuda")
    dq, dt, dc = wide(q, W + pad), torch.from_numpy(tab).cuda(), i32(ctx)
    torch.cuda.synchronize()
    c.c.window_decode_attention(layer, dq, W + pad, out, W + 16, dc, dt, tab.shape[1], len(ctx), max_ctx or max(max(ctx) + 1, 1), window, sinks)
    c.c.sync(1)
    out = out.cpu()
    assert bool(torch.isnan(out[:, W:]).all())   # beside the rows
    return out[:, :W].view(len(ctx), c.Hq, c.hd)


def expect(c, tab, r, pos, q, window, sinks, layer=0):
    return R.attention(q, *c.tokens(tab[r], R.window_keys(pos, window, sinks), layer))


def check_decode(name, c, tab, ctx, window, sinks, q, got, rows=None):
    for i, pos in enumerate(ctx):
        if pos < 0:
            assert bool((got[i] == 0).all()), (name, i)
        elif rows is None or i in rows:
            R.held(f"{name} row {i} at {pos}", got[i], *expect(c, tab, i, pos, q[i], window, sinks))


@pytest.mark.parametrize("heads", R.HEADS, ids=str)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (16, 16), (17, 4), (64, 0), (100, 33), (1000, 7), (2 ** 31 - 1, 0), (7, 2 ** 31 - 1)])
def test_decode_rows(heads, window, sinks):
    ctx = [0, 15, -1, 16, 17, 63, 64, 99, 131, 200, 299, 40]
    c = Step(heads, sum(c // 16 + 1 for c in ctx) + 2, max_batch=len(ctx), max_context=400, seed=1)
    tab = c.tables([n + 1 for n in ctx])
    q = c.queries(len(ctx))
    got = decode(c, tab, ctx, window, sinks, q)
    check_decode(f"{heads} {window}+{sinks}", c, tab, ctx, window, sinks, q, got)
    c.c.destroy()


@pytest.mark.parametrize("heads,batch,ctx,window,sinks", [
    ((8, 2, 128), 1, 5000, 4000, 4),      # one row, its keys in pieces
    ((4, 4, 64), 3, 3500, 2048, 0),
    ((16, 1, 128), 2, 4000, 4096, 16),
    ((8, 8, 64), 70, 700, 512, 5),        # more workgroups than compute units
    ((32, 8, 128), 40, 600, 333, 1),
], ids=str)
def test_decode_rows_of_long_contexts(heads, batch, ctx, window, sinks):
    lens = [ctx - 7 * i for i in range(batch)]
    c = Step(heads, sum(n // 16 + 1 for n in lens), max_batch=batch, max_context=8192, seed=2)
    tab = c.tables([n + 1 for n in lens])
    q = c.queries(batch)
    got = decode(c, tab, lens, window, sinks, q, max_ctx=ctx + 1)
    check_decode(f"{heads} x {batch}", c, tab, lens, window, sinks, q, got, rows={0, 1, batch // 2, batch - 1})
    again = decode(c, tab, lens, window, sinks, q, max_ctx=ctx + 1)
    assert torch.equal(got, again)
    c.c.destroy()


@pytest.mark.parametrize("heads", [(8, 2, 128), (9, 3, 128), (4, 4, 64)], ids=str)
@pytest.mark.parametrize("poison", [math.nan, math.inf, -math.inf])
def test_what_a_decode_row_does_not_see_does_not_reach_it(heads, poison):
    """Keys and values outside the window and the sinks, and behind the row, hold NaN or infinities, and entries of blocks between anything."""
    ctx, window, sinks = [200, 37, 16, 150], 40, 5
    c = Step(heads, 60, max_batch=4, max_context=256, seed=3)
    tab = c.tables([n + 1 for n in ctx])
    q = c.queries(4)
    for r, pos in enumerate(ctx):
        seen = set(R.window_keys(pos, window, sinks).tolist())
        for t in range(16 * (pos // 16 + 1)):
            if t not in seen:
                c.k[0, tab[r, t // 16], t % 16] = poison
                c.v[0, tab[r, t // 16], t % 16] = poison
    c.push()
    given = tab.copy()
    for r, pos in enumerate(ctx):
        for b in range(1, max((pos - window + 1) // 16, 1)):
            given[r, b] = [-7, 2 ** 31 - 1, c.n_blocks][b % 3]
    got = decode(c, given, ctx, window, sinks, q)
    check_decode(f"{heads} {poison}", c, tab, ctx, window, sinks, q, got)
    c.c.destroy()


def test_values_that_are_seen_and_not_finite_show():
    c = Step((8, 2, 128), 20, max_batch=2, max_context=256, seed=4)
    ctx = [100, 100]
    tab = c.tables([101, 101])
    q = c.queries(2)
    c.v[0, tab[0, 5], 4, 1, 7] = math.inf       # token 84 of request 0, kv head 1
    c.k[0, tab[1, 5], 4, 0, 7] = math.nan       # token 84 of request 1, kv head 0
    c.push()
    got = decode(c, tab, ctx, 50, 4, q)
    assert bool((got[0, 4:, 7] == math.inf).all()) and bool(torch.isnan(got[1, :4]).all())
    got[0, 4:, 7] = 0.0
    assert bool(torch.isfinite(got[0]).all()) and bool(torch.isfinite(got[1, 4:]).all())
    R.held("other heads", got[0, :4], *[x[:4] for x in expect(c, tab, 0, 100, q[0], 50, 4)])
    c.c.destroy()


@pytest.mark.parametrize("heads,ctx,batch", [((8, 2, 128), 150, 3), ((4, 4, 64), 3000, 1)], ids=str)
def test_blocks_that_are_none_and_lengths_out_of_range(heads, ctx, batch):
    c = Step(heads, batch * (ctx // 16 + 1) + 3, max_batch=batch + 2, max_context=4096, seed=5)
    tab = c.tables([ctx + 1] * batch + [1, 1])
    q = c.queries(batch + 2)
    bad = tab.copy()
    bad[0, ctx // 16 - 1], bad[0, ctx // 16 - 3] = c.n_blocks, -2
    lens = [ctx] * batch + [-2, 4096]
    W = c.Hq * c.hd
    out = torch.full((batch + 2, W), math.nan, dtype=torch.bfloat16, device="cuda")
    dq, dt, dc = wide(q, W), torch.from_numpy(bad).cuda(), i32(lens)
    torch.cuda.synchronize()
    c.c.window_decode_attention(0, dq, W, out, W, dc, dt, tab.shape[1], batch + 2, ctx + 1, 100, 20)
    with pytest.raises(rs.RapidServeError) as e:
        c.c.sync(1)
    assert e.value.code == rs.RS_ERR_BAD_BLOCK
    c.c.sync(1)   # once
    got = out.cpu().view(-1, c.Hq, c.hd)
    keys = np.array([j for j in R.window_keys(ctx, 100, 20) if j // 16 not in (ctx // 16 - 1, ctx // 16 - 3)])
    R.held("over what is left", got[0], *R.attention(q[0], *c.tokens(tab[0], keys)))
    for r in range(1, batch):
        R.held("others", got[r], *expect(c, tab, r, ctx, q[r], 100, 20))
    assert bool((got[batch:] == 0).all())
    c.c.destroy()


def prefill(c, tab, lens, starts, window, sinks, q, pad=8):
    W, cu = c.Hq * c.hd, [0] + [int(x) for x in np.cumsum(lens)]
    out = torch.full((cu[-1] + 2, W + 8), math.nan, dtype=torch.bfloat16, device="cuda")
    dq, dt = wide(q, W + pad), torch.from_numpy(tab).cuda()
    torch.cuda.synchronize()
    c.c.window_prefill_attention(0, dq, W + pad, out, W + 8, cu, starts, dt, tab.shape[1], window, sinks)
    c.c.sync(0)
    out = out.cpu()
    assert bool(torch.isnan(out[:, W:]).all()) and bool(torch.isnan(out[cu[-1]:]).all())
    return out[:cu[-1], :W].view(-1, c.Hq, c.hd)


def check_prefill(name, c, tab, lens, starts, window, sinks, q, got, some=None):
    at = 0
    for r, n in enumerate(lens):
        rows = [i for i in range(n) if n <= 40 or some is None or i % some == 0 or i in (1, 15, 16, n - 2, n - 1)]
        want = [expect(c, tab, r, starts[r] + i, q[at + i], window, sinks) for i in rows]
        if rows:
            R.held(f"{name} request {r}", got[[at + i for i in rows]], torch.stack([w for w, _ in want]), torch.stack([b for _, b in want]))
        at += n


@pytest.mark.parametrize("heads", R.HEADS, ids=str)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 2), (16, 4), (33, 0), (50, 20), (2 ** 31 - 1, 0), (9, 2 ** 31 - 1)])
def test_prompt_rows(heads, window, sinks):
    lens, starts = [37, 0, 1, 130, 16], [5, 9, 0, 0, 112]
    total = [s + n for s, n in zip(starts, lens)]
    c = Step(heads, sum(-(-n // 16) for n in total) + 1, max_prefill=sum(lens), max_context=400, seed=6)
    tab = c.tables(total)
    q = c.queries(sum(lens))
    got = prefill(c, tab, lens, starts, window, sinks, q)
    check_prefill(f"{heads} {window}+{sinks}", c, tab, lens, starts, window, sinks, q, got, some=7)
    c.c.destroy()


@pytest.mark.parametrize("heads,lens,starts,window,sinks", [
    ((8, 2, 128), [19], [4000], 3500, 4),          # few rows, keys in pieces
    ((4, 4, 64), [700, 33], [100, 2000], 256, 16),
    ((64, 8, 128), [900], [77], 128, 3),           # a workgroup a unit
    ((16, 16, 64), [600], [0], 100, 0),
], ids=str)
def test_prompt_rows_of_long_contexts(heads, lens, starts, window, sinks):
    total = [s + n for s, n in zip(starts, lens)]
    c = Step(heads, sum(-(-n // 16) for n in total) + 1, max_prefill=sum(lens), max_context=8192, seed=7)
    tab = c.tables(total)
    q = c.queries(sum(lens))
    got = prefill(c, tab, lens, starts, window, sinks, q)
    check_prefill(f"{heads}", c, tab, lens, starts, window, sinks, q, got, some=211)
    assert torch.equal(got, prefill(c, tab, lens, starts, window, sinks, q))
    c.c.destroy()


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64), (9, 3, 128)], ids=str)
def test_what_a_prompt_row_does_not_see_does_not_reach_it(heads):
    """Values of one token are infinite, keys of another NaN: rows before them and rows whose window has passed them are as if they were not."""
    lens, starts, window, sinks = [100], [30], 20, 3
    c = Step(heads, 12, max_prefill=100, max_context=256, seed=8)
    tab = c.tables([130])
    q = c.queries(100)
    c.v[0, tab[0, 60 // 16], 60 % 16] = math.inf
    c.k[0, tab[0, 90 // 16], 90 % 16] = math.nan
    c.v[0, tab[0, 125 // 16], 125 % 16] = math.nan
    c.push()
    got = prefill(c, tab, lens, starts, window, sinks, q)
    for i in range(100):
        pos = 30 + i
        sees = [t for t in (60, 90, 125) if pos - window < t <= pos]
        if not sees:
            R.held(f"row at {pos}", got[i], *expect(c, tab, 0, pos, q[i], window, sinks))
        elif 60 in sees and 90 not in sees:
            assert bool((got[i] == math.inf).all()), pos
        else:
            assert bool(torch.isnan(got[i]).all()), pos
    c.c.destroy()


def test_blocks_behind_four_gib():
    """The last blocks of pools of 4.3 GB each; everything before them is left unwritten."""
    heads, n_blocks = (8, 8, 128), 132000
    kp, vp = (torch.empty(n_blocks, *s, dtype=torch.bfloat16, device="cuda") for s in ((8, 4, 4, 16, 8), (8, 128, 16)))
    c = Step(heads, 24, max_batch=1, max_prefill=20, max_context=400, seed=9)
    near = c.c
    c.c = rs.Context(d_model=256, n_q_heads=8, n_kv_heads=8, head_dim=128, ffn_dim=256, n_layers=1, rms_eps=1e-5, rope_base=1e4, max_pos=64, n_blocks=n_blocks,
                     k_pool=kp, v_pool=vp, max_prefill_tokens=20, max_decode_batch=1, max_context=400)
    kp[-24:], vp[-24:] = c.kp[0], c.vp[0]
    tab = c.tables([371])
    q = c.queries(20)
    far = np.where(tab >= 0, tab + n_blocks - 24, tab).astype(np.int32)
    got = decode(c, far, [370], 200, 5, q[:1])
    check_decode("decode", c, tab, [370], 200, 5, q, got)
    got = prefill(c, far, [20], [351], 200, 5, q)
    check_prefill("prompt", c, tab, [20], [351], 200, 5, q, got)
    c.c.destroy(), near.destroy()


@pytest.mark.parametrize("ctx", [[200, 40], [3000, 2900]])   # whole rows, and keys in pieces
def test_decode_recorded_into_graphs_that_share_the_workspace(ctx):
    c = Step((8, 2, 128), 400, max_batch=2, max_context=4096, seed=10)
    tab = c.tables([n + 9 for n in ctx])
    W = 1024
    dt, dc = torch.from_numpy(tab).cuda(), i32(ctx)
    qs = [wide(c.queries(2), W) for _ in range(2)]
    outs = [torch.zeros(2, W, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    call = lambda i: c.c.window_decode_attention(0, qs[i], W, outs[i], W, dc, dt, tab.shape[1], 2, max(ctx) + 9, 2000 + i, 4)
    stream = torch.cuda.ExternalStream(c.c.get_stream(1))
    graphs = []
    torch.cuda.synchronize()
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i], stream=stream):
            call(i)
    for rep in range(4):
        for i in range(2):
            qs[i].copy_(wide(c.queries(2), W))
        dc.add_(1)
        torch.cuda.synchronize()
        for i in range(2):
            call(i)
        c.c.sync(1)
        want = [o.cpu() for o in outs]
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for g in graphs:
                g.replay()
        c.c.sync(1)
        for a, b in zip(want, outs):
            assert torch.equal(a, b.cpu()) and float(a.abs().sum()) > 0, rep
    pos = int(dc[0])
    R.held("last", outs[0][0].cpu().view(8, 128), *expect(c, tab, 0, pos, qs[0][0].cpu().view(8, 128), 2000, 4))
    del graphs
    c.c.destroy()


def test_a_partition_gives_the_same_bits():
    c = Step((8, 2, 128), 500, max_batch=4, max_prefill=150, max_context=4096, seed=11)
    ctx = [1900, 1800, 5, 700]
    tab = c.tables([n + 1 for n in ctx])
    q = c.queries(150)
    got = []
    for split in ((256, 256), (128, 128), (224, 32)):
        c.c.set_cu_split(*split)
        got.append((decode(c, tab, ctx, 1500, 4, q[:4]), prefill(c, tab[:1], [150], [1700], 900, 4, q)))
    for d, p in got[1:]:
        assert torch.equal(d, got[0][0]) and torch.equal(p, got[0][1])
    c.c.destroy()
