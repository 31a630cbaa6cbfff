"""Layer passes, captured steps and closed-loop generation over a KV cache held in 4 bits: every stage against the oracle's routine
for it, fed the operands that the stage itself read."""
import time

import numpy as np
import pytest
import torch

import oracle
import paper_2601_11822_amd as rs
import rs_synth as S
from tests import kv4_ref as R
from tests.gpu_util import TOL, Rig, check_stages_own_operands, check_tensor, to_bits, to_dev
from tests.test_gpu_tokens import _serve

pytestmark = pytest.mark.gpu


class Kv4Rig(Rig):
    """Rig over a 4-bit pool, with the pool by the definition (ref) on the host."""

    def __init__(self, shape, n_blocks, max_prefill_tokens, max_decode_batch, max_context, n_layers=1, with_oracle=True):
        self.shape, self.n_blocks, self.n_layers = shape, n_blocks, n_layers
        self.ref = np.full((n_layers, n_blocks, shape.n_kv_heads, 17 * shape.head_dim), 0xFF, np.uint8)
        self.pool = torch.from_numpy(self.ref.copy()).cuda()
        self.ctx = rs.Context.from_shape(shape, n_layers=n_layers, max_pos=max(max_context, max_prefill_tokens), n_blocks=n_blocks,
                                         kv4_pool=self.pool, max_prefill_tokens=max_prefill_tokens, max_decode_batch=max_decode_batch,
                                         max_context=max_context, device=0)
        self.wbits, self.wdev, self.olayers, self._keep = [], [], [], []
        for l in range(n_layers):
            wb = S.layer_weights(shape, l)
            wd = {k: to_dev(v) for k, v in wb.items()}
            self.ctx.set_weights(l, wd["g1"], wd["wqkv"], wd["wo"], wd["g2"], wd["wg"], wd["wu"], wd["wd"])
            self.wbits.append(wb); self.wdev.append(wd)
            if with_oracle:
                self.olayers.append(oracle.OracleLayer.from_shape(shape, wb))

    def _logical(self, layer, which):
        got = self.pool[layer].cpu().numpy()
        sh = (self.n_blocks, 16, self.shape.n_kv_heads, self.shape.head_dim)
        out = np.zeros(sh, np.uint16)
        for b in range(self.n_blocks):
            for t in range(16):
                out[b, t] = R.to_bf16_bits(R.get(got, self.shape.head_dim, b, t)[which])
        return out

    def k_bits_logical(self, layer=0):
        return self._logical(layer, 0)

    def v_bits_logical(self, layer=0):
        return self._logical(layer, 1)

    def check_to_attention(self, side, x_bits, pos, tabs, layer=0):
        """A pass whose row i sat at position pos[i] of the request with blocks tabs[i]: the rotated q, k and v of the rows; the
        bytes of the whole pool, which are the definition's of those k and v and otherwise as before; attention over the values
        that the bytes stand for."""
        sh, L, M = self.shape, self.olayers[layer], len(pos)
        x = S.bf16_bits_to_f32(x_bits)
        pos = np.asarray(pos, np.int32)
        qkv_bits = self.ctx.debug_read_workspace(side, 1, (M, sh.qkv_dim))
        qkv, heads = S.bf16_bits_to_f32(qkv_bits), sh.n_q_heads + sh.n_kv_heads
        want = L.project("wqkv", L.norm(1, x)).reshape(M, -1, sh.head_dim)
        want[:, :heads] = oracle.rope(want[:, :heads], pos, sh.rope_base)
        check_tensor("rotated q, k and v", qkv, want.reshape(M, -1))
        kv = R.f64(qkv_bits.reshape(M, -1, sh.head_dim)[:, sh.n_q_heads:])
        for i in range(M):
            R.put(self.ref[layer], sh.head_dim, tabs[i][pos[i] // 16], pos[i] % 16, kv[i, :sh.n_kv_heads], kv[i, sh.n_kv_heads:])
        assert np.array_equal(self.pool.cpu().numpy(), self.ref)
        k, v = (S.bf16_bits_to_f32(b) for b in (self.k_bits_logical(layer), self.v_bits_logical(layer)))
        attn = oracle.attn_paged(qkv.reshape(M, -1, sh.head_dim)[:, :sh.n_q_heads], k, v, np.asarray(tabs, np.int32), pos + 1)
        check_tensor("attention over the cache", S.bf16_bits_to_f32(self.ctx.debug_read_workspace(side, 2, (M, sh.q_dim))), attn.reshape(M, -1))

    def check(self, side, x_bits, y_bits, pos, tabs, layer=0):
        """The same, and what follows attention."""
        self.check_to_attention(side, x_bits, pos, tabs, layer)
        check_stages_own_operands(self, side, self.olayers[layer], len(pos), S.bf16_bits_to_f32(x_bits), y_bits, ctx=np.asarray(pos, np.int32),
                                  tables=np.asarray(tabs, np.int32), layer=layer)


def runs(cu, start, tables):
    """Position and table row of every row of a prompt pass."""
    pos = np.concatenate([np.arange(cu[r + 1] - cu[r]) + (start[r] if start is not None else 0) for r in range(len(cu) - 1)])
    return pos, np.repeat(np.asarray(tables), np.diff(cu), axis=0)


@pytest.mark.parametrize("shape", [S.TINY, S.MID, S.ODD], ids=lambda s: s.name)
@pytest.mark.parametrize("lens", [[1], [3, 1], [37, 64, 5], [300]], ids=str)
def test_prefill_then_decode_then_hybrid(shape, lens):
    """Prompts, two decode steps over them, then the next chunk of one of them beside decode rows of the others: passes small enough
    to stream the weights, of up to 64 rows and larger ones."""
    n, B = len(lens), len(lens)
    lens = np.array(lens)
    room = [int(l) + 120 for l in lens]
    n_blocks = sum(S.blocks_for(c) for c in room) + 3
    tabs = S.shuffled_block_tables(room, n_blocks, stream=5)
    rig = Kv4Rig(shape, n_blocks, max(400, int(lens.sum())), B + 1, 512)
    try:
        cu = np.concatenate([[0], np.cumsum(lens)])
        x = S.hidden_states(int(cu[-1]), shape.d_model, stream=1)
        y = rig.prefill(x, cu, tabs)
        rig.check(rs.RS_SIDE_PREFILL, x, y, *runs(cu, None, tabs))
        ctx = lens.copy()
        for step in range(2):
            x = S.hidden_states(B, shape.d_model, stream=10 + step)
            y = rig.decode(x, ctx, tabs, max_ctx=16 * tabs.shape[1] if step else None)
            rig.check(rs.RS_SIDE_DECODE, x, y, ctx, tabs)
            ctx += 1
        # a chunk behind the whole blocks of request 0 (it writes over the rest), the others decode
        start = int(ctx[0]) // 16 * 16
        for chunk in (2, 50, 90):
            x = S.hidden_states(chunk + B - 1, shape.d_model, stream=20 + chunk)
            hcu = [0, chunk]
            y = rig.hybrid(x, hcu, [start], tabs[:1], ctx[1:] if B > 1 else None, tabs[1:] if B > 1 else None)
            pos, rows = runs(hcu, [start], tabs[:1])
            rig.check(rs.RS_SIDE_PREFILL, x, y, np.concatenate([pos, ctx[1:]]), np.concatenate([rows, tabs[1:]]))
            ctx[1:] += 1
    finally:
        rig.close()


def test_layers_with_a_sparse_feed_forward_block():
    """Of two layers one is sparse: its cache, in the second layer's part of the pool, and its attention."""
    shape, lens = S.WIDE, [40, 70]
    tabs = S.shuffled_block_tables([60, 90], 16, stream=3)
    rig = Kv4Rig(shape, 16, 128, 2, 128, n_layers=2)
    try:
        g = np.random.default_rng(4)
        rnd = lambda *s: to_dev(R.to_bf16_bits((0.05 * g.standard_normal(s)).astype(np.float32)))
        d, f = shape.d_model, shape.ffn_dim
        keep = (rnd(4, d), rnd(4, f, d), rnd(4, f, d), rnd(4, d, f))
        rig.ctx.set_moe_weights(1, *keep, 4)
        for layer in (0, 1):
            x = S.hidden_states(110, d, stream=30 + layer)
            y = rig.prefill(x, [0, 40, 110], tabs, layer=layer)
            rig.check_to_attention(rs.RS_SIDE_PREFILL, x, *runs([0, 40, 110], None, tabs), layer=layer)
            x = S.hidden_states(2, d, stream=40 + layer)
            z = rig.decode(x, lens, tabs, layer=layer)
            rig.check_to_attention(rs.RS_SIDE_DECODE, x, lens, tabs, layer=layer)
            assert np.isfinite(S.bf16_bits_to_f32(y)).all() and np.isfinite(S.bf16_bits_to_f32(z)).all()
    finally:
        rig.close()


def test_captured_step_is_the_eager_one_over_replays():
    """rs_decode_layer_graph over a cache in 4 bits: contexts that grow, another partition (another capture), a prompt's pass on the
    other side in between; outputs and the whole pool equal those of the eager calls to the bit."""
    shape, B, bucket, pre_T = S.MID, 5, 1024, 256
    ctx0 = np.array([30, 500, 511, 64, 700], np.int32)
    n_blocks = B * S.blocks_for(bucket) + S.blocks_for(pre_T) + 8
    tabs = S.shuffled_block_tables([bucket] * B + [pre_T], n_blocks, stream=7)
    pre_x = S.hidden_states(pre_T, shape.d_model, stream=71)
    held = np.random.default_rng(1).integers(0, 256, (1, n_blocks, shape.n_kv_heads, 17 * shape.head_dim), dtype=np.uint8)
    held[..., 16 * shape.head_dim:] = held[..., 16 * shape.head_dim:] % 8 + 122   # scales of 2^-5 to 4

    def run(graphed):
        rig = Kv4Rig(shape, n_blocks, pre_T, B, bucket, with_oracle=False)
        outs = []
        try:
            rig.pool.copy_(torch.from_numpy(held))
            x = to_dev(S.hidden_states(B, shape.d_model, stream=80)); y = torch.empty_like(x)
            cl, tab = torch.from_numpy(ctx0.copy()).cuda(), torch.from_numpy(np.ascontiguousarray(tabs[:B])).cuda()
            ptab = torch.from_numpy(np.ascontiguousarray(tabs[B:])).cuda()
            px = to_dev(pre_x); py = torch.empty_like(px)
            c = rig.ctx
            for s in range(5):
                if s == 3:
                    c.set_cu_split(192, 64)
                x.copy_(to_dev(S.hidden_states(B, shape.d_model, stream=80 + s)))
                cl.copy_(torch.from_numpy(ctx0 + s).cuda())
                torch.cuda.synchronize()
                if s % 2 == 1:
                    c.prefill_layer(0, px, py, [0, pre_T], ptab, tab.shape[1])
                (c.decode_layer_graph if graphed else c.decode_layer)(0, x, y, cl, tab, tab.shape[1], B, bucket)
                c.sync(rs.RS_SIDE_DECODE); c.sync(rs.RS_SIDE_PREFILL)
                outs += [to_bits(y).copy(), to_bits(py).copy() if s % 2 == 1 else np.zeros(1), rig.pool.cpu().numpy()]
        finally:
            rig.close()
        return outs

    eager, graphed = run(False), run(True)
    for i, (a, b) in enumerate(zip(eager, graphed)):
        assert np.array_equal(a, b), f"item {i}"
    assert np.isfinite(S.bf16_bits_to_f32(eager[0])).all() and not np.array_equal(eager[0], eager[3])


@pytest.mark.parametrize("width", [64, 160])   # whole rows, and shares of them
def test_calls_captured_by_the_caller_and_replayed(width):
    """Append, attention and reading back recorded from the decode side's stream into one graph; two graphs, of different batch
    sizes, that share the side's workspace.  Replays with other queries, tokens and lengths are the eager calls' results to the bit."""
    Hq, Hkv, hd, n_blocks = 8, 2, 128, 1000
    g = np.random.default_rng(2)
    pool = torch.zeros((1, n_blocks, Hkv, 17 * hd), dtype=torch.uint8, device="cuda")
    c = rs.Context(d_model=256, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=hd, ffn_dim=256, n_layers=1, rms_eps=1e-5, rope_base=1e4, max_pos=64,
                   n_blocks=n_blocks, kv4_pool=pool, max_prefill_tokens=64, max_decode_batch=6, max_context=16 * width)
    held = g.integers(0, 256, tuple(pool.shape), dtype=np.uint8)
    held[..., 16 * hd:] = held[..., 16 * hd:] % 8 + 122
    pool.copy_(torch.from_numpy(held))
    tab = torch.from_numpy(g.permutation(n_blocks)[:6 * width].reshape(6, width).astype(np.int32)).cuda()
    rnd = lambda n, w: to_dev(R.to_bf16_bits(g.standard_normal((n, w)).astype(np.float32)))
    stream = torch.cuda.ExternalStream(c.get_stream(1))

    class Step:
        def __init__(self, B):
            self.B = B
            self.q, self.k, self.v = rnd(B, Hq * hd), rnd(B, Hkv * hd), rnd(B, Hkv * hd)
            self.ctx = torch.zeros(B, dtype=torch.int32, device="cuda")
            self.out = torch.zeros((B, Hq * hd), dtype=torch.bfloat16, device="cuda")
            self.back = [torch.zeros((16 * B, Hkv * hd), dtype=torch.bfloat16, device="cuda") for _ in range(2)]

        def calls(self):
            B = self.B
            c.kv4_append(1, 0, self.k, self.v, Hkv * hd, self.ctx, tab, width, B)
            c.kv4_decode_attention(0, self.q, Hq * hd, self.out, Hq * hd, self.ctx, tab, width, B, 16 * width)
            c.kv4_read(1, 0, self.back[0], self.back[1], Hkv * hd, [16 * i for i in range(B + 1)], [32] * B, tab, width)

        def change(self):
            self.q.copy_(rnd(self.B, Hq * hd)), self.k.copy_(rnd(self.B, Hkv * hd)), self.v.copy_(rnd(self.B, Hkv * hd))
            self.ctx.copy_(torch.from_numpy(g.integers(32, 16 * width, self.B).astype(np.int32)))
            self.ctx[g.integers(self.B)] = -1 if g.random() < 0.3 else 32

        def results(self):
            return [to_bits(self.out).copy(), to_bits(self.back[0]).copy(), to_bits(self.back[1]).copy(), pool.cpu().numpy()]

    steps = [Step(1), Step(6)]
    graphs = []
    torch.cuda.synchronize()
    for s in steps:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            s.calls()
        graphs.append(graph)
    for rep in range(6):
        for s, graph in zip(steps, graphs):
            s.change()
            before = pool.clone()
            torch.cuda.synchronize()
            s.calls()
            c.sync(1)
            want = s.results()
            pool.copy_(before)
            for t in [s.out] + s.back:
                t.zero_()
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                graph.replay()
            c.sync(1)
            for a, b in zip(want, s.results()):
                assert np.array_equal(a, b), (rep, s.B)
    del graphs
    c.destroy()


def test_two_contexts_at_once_and_both_sides_of_one():
    """Prompts on one context's prefill side, decode steps on its decode side and on another context's, without waits in between:
    each result is that of the call made alone, to the bit."""
    def fresh(heads, seed):
        Hq, Hkv, hd = heads
        g = np.random.default_rng(seed)
        pool = torch.zeros((1, 700, Hkv, 17 * hd), dtype=torch.uint8, device="cuda")
        held = g.integers(0, 256, tuple(pool.shape), dtype=np.uint8)
        held[..., 16 * hd:] = held[..., 16 * hd:] % 8 + 122
        pool.copy_(torch.from_numpy(held))
        c = rs.Context(d_model=256, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=hd, ffn_dim=256, n_layers=1, rms_eps=1e-5, rope_base=1e4, max_pos=64,
                       n_blocks=700, kv4_pool=pool, max_prefill_tokens=512, max_decode_batch=16, max_context=4096)
        tab = torch.from_numpy(np.stack([g.permutation(700)[:256] for _ in range(16)]).astype(np.int32)).cuda()
        q = to_dev(R.to_bf16_bits(g.standard_normal((512, Hq * hd)).astype(np.float32)))
        ctx = torch.from_numpy(g.integers(0, 4090, 16).astype(np.int32)).cuda()
        return c, q, tab, ctx, Hq * hd

    def prompts(c, q, tab, ctx, W, start):
        return lambda o: c.kv4_prefill_attention(0, q, W, o, W, [0, 300, 512], [start, 0], tab, 256)

    def step(c, q, tab, ctx, W, max_ctx):
        return lambda o: c.kv4_decode_attention(0, q, W, o, W, ctx, tab, 256, 16, max_ctx)

    pair = [fresh((8, 2, 128), 1), fresh((4, 4, 64), 2)]
    jobs = []
    for one in pair:
        c, q = one[:2]
        jobs += [(c, 0, q, prompts(*one, 0)), (c, 0, q, prompts(*one, 1800)), (c, 1, q[:16], step(*one, 4096)), (c, 1, q[:16], step(*one, 4090))]
    alone = []
    for c, side, q, f in jobs:
        o = torch.zeros_like(q)
        torch.cuda.synchronize()
        f(o)
        c.sync(side)
        alone.append(to_bits(o).copy())
    for rep in range(3):
        outs = [torch.zeros_like(q) for _, _, q, _ in jobs]
        torch.cuda.synchronize()
        for (c, side, q, f), o in zip(jobs, outs):
            f(o)
        for c, *_ in pair:
            c.sync(0), c.sync(1)
        for o, want in zip(outs, alone):
            assert np.array_equal(to_bits(o), want)
    for c, *_ in pair:
        c.destroy()


# ------------------------------------------------------------------------------ closed loop
VOCAB = 1000
PROMPTS = [(1, 37, 30, 0), (2, 5, 40, 0), (3, 64, 25, 2), (4, 16, 3, 3), (5, 23, 33, 6)]


def head(rig):
    hb = S.head_weights(rig.shape.d_model, VOCAB)
    hd = {k: to_dev(v) for k, v in hb.items()}
    rig.ctx.set_head(hd["embed"], hd["final_norm"], hd["lm_head"], VOCAB, -1)
    rig._keep.append(hd)


def follow(shape, n_layers, requests, outs):
    """The loop's tokens fed to the same library's single calls, one request at a time (whole prompt, then a row a step): each token
    must be a near-maximum of the logits there, and their only one where they decide by more than rounding may move them."""
    rig = Kv4Rig(shape, 16, 128, 1, 128, n_layers=n_layers, with_oracle=False)
    same = total = 0
    try:
        head(rig)
        c = rig.ctx
        tab = torch.arange(8, dtype=torch.int32, device="cuda").reshape(1, 8)
        for rid, prompt, mn, _ in requests:
            got = outs[rid]
            assert len(got) == mn
            for k in range(mn):
                side = rs.RS_SIDE_DECODE if k else rs.RS_SIDE_PREFILL
                toks = torch.from_numpy(np.asarray([got[k - 1]] if k else prompt, np.int32)).cuda()
                n = len(toks)
                x = torch.zeros((n, shape.d_model), dtype=torch.bfloat16, device="cuda")
                logits, tok = torch.zeros((n, VOCAB), dtype=torch.float32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
                pos = torch.tensor([len(prompt) + k - 1], dtype=torch.int32, device="cuda")
                torch.cuda.synchronize()
                c.embed(side, toks, n, x)
                y = torch.zeros_like(x)
                torch.cuda.synchronize()
                for l in range(n_layers):
                    if k:
                        c.decode_layer(l, x, y, pos, tab, 8, 1, len(prompt) + k)
                    else:
                        c.prefill_layer(l, x, y, [0, n], tab, 8)
                    x, y = y, x
                c.lm_head_greedy(side, x, n, logits, tok)
                c.sync(side)
                lg = logits[-1].cpu().numpy()
                slack = 2 * TOL * np.max(np.abs(lg))
                assert lg[got[k]] >= lg.max() - slack, f"request {rid} token {k}"
                same += int(np.argmax(lg)) == got[k]
                total += 1
    finally:
        rig.close()
    return same / total


@pytest.mark.parametrize("mode", ["graphs", "eager", "hybrid", "few blocks", "engine"])
def test_closed_loop(mode):
    shape, n_layers = S.TINY, 2
    few = mode == "few blocks"
    prompts = [(1, 20, 40, 0), (2, 20, 40, 0)] if few else PROMPTS
    requests = [(rid, S.prompt_tokens(pl, VOCAB, rid), mn, arr) for rid, pl, mn, arr in prompts]
    rig = Kv4Rig(shape, 7 if few else 64, 128, 4, 128, n_layers=n_layers, with_oracle=False)
    try:
        head(rig)
        c = rig.ctx
        if mode == "hybrid":
            c.set_hybrid_batching(48)
        c.set_step_graphs(mode == "graphs")
        if mode == "engine":
            c.engine_start()
            for rid, prompt, mn, _ in requests:
                c.submit_tokens(rid, prompt, mn)
            until = time.time() + 60
            while c.engine_stats()["finished"] < len(requests):
                assert time.time() < until, c.engine_stats()
                time.sleep(0.01)
            c.engine_stop(drain=True)
            outs = {rid: c.request_output(rid)[0].tolist() for rid, *_ in requests}
        else:
            outs, preempted = _serve(rig, None, VOCAB, -1, requests, wait=False)
            assert (preempted > 0) == few
        assert (c.step_graph_stats()[1] > 0) == (mode == "graphs")
        assert c.kv_num_free() == rig.n_blocks
    finally:
        rig.close()
    frac = follow(shape, n_layers, requests, outs)
    print(f"  {mode}: {frac:.2%} of the tokens are the single calls' own choice", flush=True)
    assert frac >= 0.9


def test_what_a_cache_in_4_bits_is_not_served_by():
    rig = Kv4Rig(S.TINY, 8, 32, 4, 64, with_oracle=False)
    try:
        x = to_dev(S.hidden_states(2, S.TINY.d_model, stream=5)); y = torch.zeros_like(x)
        cl, tab = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.arange(8, dtype=torch.int32, device="cuda").reshape(2, 4)
        torch.cuda.synchronize()
        with pytest.raises(rs.RapidServeError) as e:
            rig.ctx.decode_layer_noalloc(0, x, y, cl, tab, 4, 2, 64)
        assert e.value.code == rs.RS_ERR_STATE
        rig.ctx.sync(1)
        assert (y == 0).all() and (rig.pool == 0xFF).all()
    finally:
        rig.close()
