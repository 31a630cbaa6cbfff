"""Steps of speculative decoding as a program makes them: plan, store and tree attention in every layer, a path chosen, compact; then the window over
what was accepted.  Eager against the definitions, and recorded into a graph against eager, to the bit."""
import numpy as np
import pytest
import torch

import paper_2601_11822_amd as rs
from tests import step_ref as R
from tests.step_ref import Step, i32, wide

pytestmark = pytest.mark.gpu

B, DRAFT, LAYERS, ROWS = 4, 12, 2, 40


class Server:
    """Everything on the GPU but the choice of the path: lengths, tables, the stack of free blocks."""

    def __init__(self, heads, seed):
        self.s = s = Step(heads, 60, max_batch=B, max_prefill=B, max_context=400, n_layers=LAYERS, seed=seed, max_pos=400)
        self.ctx = [20, 0, -1, 37]
        self.tab = s.tables([max(n, 0) for n in self.ctx], width=25)
        self.held = [-(-max(n, 0) // 16) for n in self.ctx]
        self.free = s.rest
        W = (s.Hq + 2 * s.Hkv) * s.hd
        self.Wq, self.W = s.Hq * s.hd, W
        self.d = dict(lens=i32(self.ctx), new=i32([0] * B), held=i32(self.held), tab=i32(self.tab), free=i32(self.free), n_free=i32([len(self.free)]),
                      parents=i32(np.full((B, DRAFT), -1)), cu=i32([0] * (B + 1)), pos=i32([0] * ROWS), slots=i32([0] * ROWS), keep=i32(np.zeros((B, DRAFT))),
                      keep_lens=i32([0] * B))
        self.masks = torch.zeros(ROWS, dtype=torch.int64, device="cuda")
        self.qkv = [torch.zeros(ROWS, W, dtype=torch.bfloat16, device="cuda") for _ in range(LAYERS)]
        self.out = [torch.zeros(ROWS, self.Wq, dtype=torch.bfloat16, device="cuda") for _ in range(LAYERS)]
        self.win = torch.zeros(B, self.Wq, dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()

    def draft(self, new, parents, qkv):
        self.d["new"].copy_(i32(new)), self.d["parents"].copy_(i32(parents))
        for mine, x in zip(self.qkv, qkv):
            mine.copy_(x)
        torch.cuda.synchronize()

    def verify(self):
        """The queries are rotated in place, in the projection's own rows."""
        d, c = self.d, self.s.c
        c.kv_plan(1, d["lens"], d["new"], d["held"], d["tab"], 25, B, d["free"], len(self.free), d["n_free"], ROWS, d["cu"], d["pos"], d["slots"], d["held"],
                  d["n_free"], parents=d["parents"], parent_stride=DRAFT, masks=self.masks)
        for layer in range(LAYERS):
            c.kv_store(1, layer, self.qkv[layer], self.W, self.qkv[layer], self.W, d["pos"], d["slots"], ROWS, n_rows=d["cu"][B:])
            c.tree_attention(layer, self.qkv[layer], self.W, self.out[layer], self.Wq, d["lens"], d["cu"], self.masks, d["tab"], 25, B, ROWS, DRAFT, 400)

    def accept(self):
        d, c = self.d, self.s.c
        c.kv_compact(1, 0, LAYERS, d["lens"], d["keep"], DRAFT, d["keep_lens"], d["tab"], 25, B)

    def look(self, ctx, q):
        self.s.c.window_decode_attention(1, q, self.Wq, self.win, self.Wq, ctx, self.d["tab"], 25, B, 400, 9, 2)

    def choose(self, keep):
        padded = np.zeros((B, DRAFT), np.int32)
        for b, k in enumerate(keep):
            padded[b, :len(k)] = k
        self.d["keep"].copy_(i32(padded)), self.d["keep_lens"].copy_(i32([len(k) for k in keep]))
        torch.cuda.synchronize()


def path_of(g, parents, n):
    """A path from a first token down, ascending, or none."""
    if n == 0 or g.random() < 0.2:
        return []
    at, path = int(g.integers(0, n)), []
    while at >= 0:
        path.append(at)
        at = int(parents[at])
    return path[::-1]


@pytest.mark.parametrize("heads", [(8, 2, 128), (9, 3, 128), (4, 4, 64)], ids=str)
def test_steps_eager_and_recorded(heads):
    g = np.random.default_rng(3)
    eager, taped = Server(heads, 5), Server(heads, 5)
    stream = torch.cuda.ExternalStream(taped.s.c.get_stream(1))
    ctx_last, q_last = [i32([-1] * B) for _ in range(2)], [torch.zeros(B, eager.Wq, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    torch.cuda.synchronize()
    with torch.cuda.graph(graphs[0], stream=stream):
        taped.verify()
    with torch.cuda.graph(graphs[1], stream=stream):
        taped.accept()
        taped.look(ctx_last[1], q_last[1])
    s = eager.s
    ctx, tab, held, free = list(eager.ctx), eager.tab, eager.held, eager.free
    for step in range(6):
        new = [int(g.integers(1, DRAFT + 1)), [0, 3, 12][step % 3], 5, int(g.integers(0, DRAFT + 1))]
        parents = np.full((B, DRAFT), -1, np.int32)
        for b in range(B):
            parents[b, :new[b]] = R.random_tree(g, new[b])
        rows = [torch.randn(ROWS, eager.W, generator=torch.Generator().manual_seed(100 * step + i)).bfloat16() for i in range(LAYERS)]
        for x in (eager, taped):
            x.draft(new, parents, rows)
        eager.verify()
        with torch.cuda.stream(stream):
            graphs[0].replay()
        s.c.sync(1), taped.s.c.sync(1)

        # the plan, and what the cache holds now
        tab, cu, pos, slots, masks, held, left = R.plan(ctx, new, held, tab, free, parents)
        free, n = free[:left], cu[-1]
        for x in (eager, taped):
            assert np.array_equal(x.d["tab"].cpu().numpy(), tab) and x.d["cu"].tolist() == cu and x.d["pos"][:n].tolist() == pos
            assert x.d["slots"][:n].tolist() == slots and x.d["n_free"].tolist() == [left] and x.d["held"].tolist() == held
        for layer in range(LAYERS):
            x = rows[layer].view(ROWS, -1, s.hd)[:n]
            at = torch.tensor(slots)
            k, v = s.pulled(layer)
            y = R.rotated(x[:, :s.Hq + s.Hkv].double(), [pos], [0] * (s.hd // 2), s.rope_base)
            e = R.rotation_bound(x[:, :s.Hq + s.Hkv].double()) * (1 + 2.0 ** -8) + 2.0 ** -8 * y.abs()
            q = eager.qkv[layer][:, :eager.Wq].cpu().view(ROWS, s.Hq, s.hd)
            R.held(f"step {step} queries", q[:n], y[:, :s.Hq], e[:, :s.Hq])
            R.held(f"step {step} keys", k[at // 16, at % 16], y[:, s.Hq:], e[:, s.Hq:])
            assert torch.equal(v[at // 16, at % 16], x[:, s.Hq + s.Hkv:])
            assert torch.equal(eager.qkv[layer][n:].cpu(), rows[layer][n:])
            s.k[layer][at // 16, at % 16], s.v[layer][at // 16, at % 16] = k[at // 16, at % 16], v[at // 16, at % 16]
            got = eager.out[layer].cpu().view(ROWS, s.Hq, s.hd)
            for b in range(B):
                for i in range(cu[b + 1] - cu[b]):
                    r = cu[b] + i
                    R.held(f"step {step} layer {layer} row {r}", got[r],
                           *R.attention(q[r], *s.tokens(tab[b], R.tree_keys(ctx[b], new[b], masks[r]), layer)))
            assert torch.equal(eager.out[layer], taped.out[layer]) and torch.equal(eager.qkv[layer], taped.qkv[layer])

        # a path is accepted
        keep = [path_of(g, parents[b], new[b] if ctx[b] >= 0 else 0) for b in range(B)]
        before, last = list(ctx), [c + len(k) - 1 if c >= 0 else -1 for c, k in zip(ctx, keep)]
        q = torch.randn(B, eager.Wq, generator=torch.Generator().manual_seed(7 + step)).bfloat16()
        for i, x in enumerate((eager, taped)):
            x.choose(keep)
            ctx_last[i].copy_(i32(last)), q_last[i].copy_(q)
        torch.cuda.synchronize()
        eager.accept()
        eager.look(ctx_last[0], q_last[0])
        with torch.cuda.stream(stream):
            graphs[1].replay()
        s.c.sync(1), taped.s.c.sync(1)
        for b, kept in enumerate(keep):
            for i, t in enumerate(kept):
                a, z = before[b] + t, before[b] + i
                for layer in range(LAYERS):
                    for p in (s.k[layer], s.v[layer]):
                        p[tab[b, z // 16], z % 16] = p[tab[b, a // 16], a % 16]
        for layer in range(LAYERS):
            for x in (s, taped.s):
                k, v = x.pulled(layer)
                assert torch.equal(k, s.k[layer]) and torch.equal(v, s.v[layer])
        assert torch.equal(eager.win, taped.win)
        for b, p in enumerate(last):
            want = R.attention(q[b].view(s.Hq, s.hd), *s.tokens(tab[b], R.window_keys(p, 9, 2), 1)) if p >= 0 else None
            if p >= 0:
                R.held(f"step {step} window", eager.win[b].cpu().view(s.Hq, s.hd), *want)
            else:
                assert bool((eager.win[b] == 0).all())
        ctx = [c + len(k) if c >= 0 else -1 for c, k in zip(ctx, keep)]
        for x in (eager, taped):
            x.d["lens"].copy_(i32(ctx))
    assert s.c.kv_num_free() == 60   # the library's own allocator has no part in it here
    del graphs
    eager.s.c.destroy(), taped.s.c.destroy()


def test_a_step_that_finds_no_blocks_does_nothing():
    """The calls behind a plan that could not be done find no rows."""
    x = Server((8, 2, 128), 6)
    x.d["n_free"].copy_(i32([0]))
    x.draft([12, 12, 0, 12], np.full((B, DRAFT), -1), [torch.ones(ROWS, x.W).bfloat16()] * LAYERS)
    x.verify()
    with pytest.raises(rs.RapidServeError) as e:
        x.s.c.sync(1)
    assert e.value.code == rs.RS_ERR_NO_BLOCKS
    x.s.c.sync(1)
    assert x.d["cu"].tolist() == [0] * (B + 1) and x.d["held"].tolist() == x.held and bool((x.out[0] == 0).all()) and bool((x.qkv[0] == 1).all())
    for layer in range(LAYERS):
        k, v = x.s.pulled(layer)
        assert torch.equal(k, x.s.k[layer]) and torch.equal(v, x.s.v[layer])
    x.s.c.destroy()
