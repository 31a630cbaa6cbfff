"""The 4-bit cache's calls at the ends of what they take: blocks behind 4 GiB, more KV heads than shares, the most rows of a call, prompts
recorded into a graph."""
import numpy as np
import pytest
import torch

import paper_2601_11822_amd as rs
from tests import kv4_ref as R
from tests.gpu_util import to_bits, to_dev
from tests.test_gpu_kv4 import Cache, held_to, i32, run_decode, run_prefill

pytestmark = pytest.mark.gpu


def test_blocks_behind_4_gib():
    """The same requests in the first blocks of a pool of two layers and in its last ones, 8.7 GB further (4.3 of them in a layer): what is written, read back and
    computed is the same to the bit, and nothing else is written."""
    Hq, Hkv, hd, n_blocks = 8, 2, 128, 1000000
    lens, T, B = [70, 33], 103, 2
    pool = torch.full((2, n_blocks, Hkv, 17 * hd), 0xFF, dtype=torch.uint8, device="cuda")
    c = rs.Context(d_model=256, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=hd, ffn_dim=256, n_layers=2, rms_eps=1e-5, rope_base=1e4, max_pos=64,
                   n_blocks=n_blocks, kv4_pool=pool, max_prefill_tokens=128, max_decode_batch=4, max_context=9000)
    g = np.random.default_rng(3)
    W, Wq = Hkv * hd, Hq * hd
    rnd = lambda n, w: to_dev(R.to_bf16_bits(g.standard_normal((n, w)).astype(np.float32)))
    k, v, q, k1, v1, q1 = rnd(T, W), rnd(T, W), rnd(T, Wq), rnd(B, W), rnd(B, W), rnd(B, Wq)
    ctx, outs = i32(lens), []
    ids = np.array([[0, 2, 4, 6, 8, -1], [1, 3, 5, -1, -1, -1]])
    for layer, places in ((0, ids), (1, np.where(ids < 0, -1, n_blocks - 1 - ids))):
        tab = i32(np.concatenate([places, np.full((2, 594), -1)], 1))   # wide enough for whole rows and for shares
        o = [torch.zeros((T, Wq), dtype=torch.bfloat16, device="cuda")] + [torch.zeros((B, Wq), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        back = [torch.zeros((T + B, W), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        torch.cuda.synchronize()
        c.kv4_write(0, layer, k, v, W, [0, 70, 103], None, tab, 600)
        c.kv4_prefill_attention(layer, q, Wq, o[0], Wq, [0, 70, 103], None, tab, 600)
        c.sync(0)
        c.kv4_append(1, layer, k1, v1, W, ctx, tab, 600, B)
        c.kv4_decode_attention(layer, q1, Wq, o[1], Wq, ctx, tab, 600, B, 71)
        c.kv4_decode_attention(layer, q1, Wq, o[2], Wq, ctx, tab, 600, B, 9000)
        c.kv4_read(1, layer, back[0], back[1], W, [0, 71, 105], None, tab, 600)
        c.sync(1)
        outs.append([to_bits(t).copy() for t in o + back] + [pool[layer, torch.from_numpy(p[p >= 0]).cuda()].cpu().numpy() for p in places])
    for a, b in zip(*outs):
        assert np.array_equal(a, b)
    assert np.isfinite(R.f64(outs[0][0])).all() and np.isfinite(R.f64(outs[0][1])).all()
    assert (pool[0, 9:] == 0xFF).all() and (pool[1, :n_blocks - 9] == 0xFF).all()
    c.destroy()


@pytest.mark.parametrize("max_ctx", [400, 9000])
def test_more_kv_heads_than_shares(max_ctx):
    """520 KV heads: a workgroup each takes the tokens of all rows."""
    c = Cache((520, 520, 64), 26, max_batch=4, max_context=9000, seed=4)
    ctx = [299, -1, 4, 63]
    tab, _ = c.tables([n + 1 for n in ctx])
    c.ref[0] = c.g.integers(0, 256, c.ref[0].shape, dtype=np.uint8)
    c.ref[0, ..., 16 * 64:] = c.ref[0, ..., 16 * 64:] % 4 + 124
    c.pool.copy_(torch.from_numpy(c.ref))
    tab = np.concatenate([tab, np.full((4, 563), -1, np.int32)], 1)
    q = c.queries(4)
    got = run_decode(c, q, ctx, torch.from_numpy(tab).cuda(), tab.shape[1], max_ctx)
    assert (got[1] == 0).all()
    for r in (0, 2, 3):
        k, v = R.gather(c.ref[0], c.hd, tab[r], ctx[r] + 1)
        want, bound = R.attention(R.f64(q[r:r + 1]), k, v, ctx[r])
        held_to(got[r:r + 1], want, bound, f"row {r}")
    c.c.destroy()


@pytest.mark.parametrize("max_ctx", [400, 5000])
def test_the_most_rows_of_a_call(max_ctx):
    """65535 rows, of up to 399 tokens, of blocks that they share: whole rows, and shares of all their tokens."""
    B = 65535
    c = Cache((2, 1, 64), 200, max_batch=B, max_context=5000, seed=5)
    c.ref[0] = c.g.integers(0, 256, c.ref[0].shape, dtype=np.uint8)
    c.ref[0, ..., 16 * 64:] = c.ref[0, ..., 16 * 64:] % 4 + 124
    c.pool.copy_(torch.from_numpy(c.ref))
    ctx = c.g.integers(-1, 399, B)
    ctx[c.g.random(B) < 0.5] = -1
    ctx[[0, 1, B - 1]] = 398, -1, 200
    width = -(-max_ctx // 16)
    base = c.g.permutation(200).astype(np.int32)
    tab = np.full((B, width), -1, np.int32)
    tab[:, :25] = base[(np.arange(B)[:, None] * 7 + np.arange(25)) % 200]
    q = c.queries(B)
    got = run_decode(c, q, ctx, torch.from_numpy(tab).cuda(), width, max_ctx)
    assert np.isfinite(got).all() and (got[ctx < 0] == 0).all() and (np.abs(got[ctx >= 0]).max((1, 2)) > 0).all()
    rows = [0, B - 1] + [int(r) for r in c.g.choice(np.flatnonzero(ctx >= 0), 60, replace=False)]
    for r in rows:
        k, v = R.gather(c.ref[0], c.hd, tab[r], ctx[r] + 1)
        want, bound = R.attention(R.f64(q[r:r + 1]), k, v, int(ctx[r]))
        fine = bool((np.abs(got[r] - want[0]) <= bound[0]).all())
        assert fine, r
    c.c.destroy()


def test_the_most_tokens_appended_by_a_call():
    B, W = 65535, 64
    c = Cache((1, 1, 64), 4096, max_batch=1, seed=6)
    k, v = (c.g.standard_normal((B, W)).astype(np.float32) for _ in range(2))
    k, v = R.to_bf16_bits(k), R.to_bf16_bits(v)
    perm = c.g.permutation(4096).astype(np.int32)
    pos = np.arange(B) % 16
    pos[5] = -1
    dk, dv, tab, dpos = to_dev(k), to_dev(v), i32(perm[np.arange(B) // 16].reshape(B, 1)), i32(pos)
    torch.cuda.synchronize()
    c.c.kv4_append(1, 0, dk, dv, W, dpos, tab, 1, B)
    c.c.sync(1)
    kc, ks = R.quantise(R.f64(k))
    vc, vs = R.quantise(R.f64(v))
    for t in range(16):
        rows = np.arange(t, B, 16)
        rows = rows[pos[rows] >= 0]
        places = R.places(64, t)
        for (codes, scales), at, sat in (((kc, ks), places[0], places[2]), ((vc, vs), places[1], places[3])):
            blk = perm[rows // 16]
            c.ref[0, blk[:, None, None], 0, at[None]] = codes[rows][..., 0::2] | codes[rows][..., 1::2] << 4
            c.ref[0, blk[:, None], 0, sat[None]] = scales[rows]
    c.same_pool()
    c.c.destroy()


@pytest.mark.parametrize("starts", [[0, 0], [3000, 64]])   # uncut, and cut in pieces
def test_prompts_recorded_into_a_graph(starts):
    """Write, attention and reading back recorded from the prefill side's stream; replays with other rows over the same cache are the eager
    calls' results to the bit."""
    lens = [37, 20]
    held = [s + n for s, n in zip(starts, lens)]
    c = Cache((8, 2, 128), 230, max_prefill=64, max_context=4096, seed=7)
    tab, dtab = c.tables(held)
    c.ref[0] = c.g.integers(0, 256, c.ref[0].shape, dtype=np.uint8)
    c.ref[0, ..., 16 * 128:] = c.ref[0, ..., 16 * 128:] % 4 + 124
    c.pool.copy_(torch.from_numpy(c.ref))
    W, Wq, T, cu = 256, 1024, 57, [0, 37, 57]
    rnd = lambda w: to_dev(R.to_bf16_bits(c.g.standard_normal((T, w)).astype(np.float32)))
    k, v, q = rnd(W), rnd(W), rnd(Wq)
    outs = [torch.zeros((T, w), dtype=torch.bfloat16, device="cuda") for w in (Wq, W, W)]

    def calls():
        c.c.kv4_write(0, 0, k, v, W, cu, starts, dtab, tab.shape[1])
        c.c.kv4_prefill_attention(0, q, Wq, outs[0], Wq, cu, starts, dtab, tab.shape[1])
        c.c.kv4_read(0, 0, outs[1], outs[2], W, cu, starts, dtab, tab.shape[1])

    stream = torch.cuda.ExternalStream(c.c.get_stream(0))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        calls()
    for rep in range(4):
        for t, w in ((k, W), (v, W), (q, Wq)):
            t.copy_(rnd(w))
        before = c.pool.clone()
        torch.cuda.synchronize()
        calls()
        c.c.sync(0)
        want = [to_bits(t).copy() for t in outs] + [c.pool.cpu().numpy()]
        c.pool.copy_(before)
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        c.c.sync(0)
        for a, b in zip(want, [to_bits(t).copy() for t in outs] + [c.pool.cpu().numpy()]):
            assert np.array_equal(a, b), rep
        assert np.isfinite(R.f64(want[0])).all()
    del graph
    c.c.destroy()
