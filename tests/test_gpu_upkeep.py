"""Plans, writes and moves of the bf16 cache on the GPU against their definitions."""
import math

import numpy as np
import pytest
import torch

import paper_2601_11822_amd as rs
from tests import step_ref as R
from tests.step_ref import Step, i32, i64, wide

pytestmark = pytest.mark.gpu


class Plan:
    """Inputs and outputs of one plan on the GPU; rows behind the last hold -9."""

    def __init__(self, lens, new, held, tab, free, parents=None, room=5, cap=None):
        self.B, self.rows = len(lens), sum(n for n, c in zip(new, lens) if c != -1) + room
        self.lens, self.new, self.held, self.tab, self.free, self.n_free = i32(lens), i32(new), i32(held), i32(tab), i32(np.append(free, -77)), i32([len(free)])
        self.cap = len(free) if cap is None else cap
        self.parents = i32(parents) if parents is not None else None
        self.cu, self.pos, self.slots = i32([-9] * (self.B + 1)), i32([-9] * (self.rows + 3)), i32([-9] * (self.rows + 3))
        self.masks = torch.full((self.rows + 3,), -9, dtype=torch.int64, device="cuda")
        self.held_out, self.n_free_out = i32([-9] * self.B), i32([-9])

    def run(self, c, in_place=False, side=1, max_rows=None):
        torch.cuda.synchronize()
        trees = self.parents is not None
        c.c.kv_plan(side, self.lens, self.new, self.held, self.tab, self.tab.shape[1], self.B, self.free, self.cap, self.n_free,
                    self.rows if max_rows is None else max_rows, self.cu, self.pos, self.slots, self.held if in_place else self.held_out,
                    self.n_free if in_place else self.n_free_out, parents=self.parents, parent_stride=self.parents.shape[1] if trees else 0,
                    masks=self.masks if trees else None)

    def same(self, want, in_place=False):
        tab, cu, pos, slots, masks, held, left = want
        n = cu[-1]
        assert np.array_equal(self.tab.cpu().numpy(), tab) and self.cu.tolist() == cu
        assert self.pos[:n].tolist() == pos and self.slots[:n].tolist() == slots
        assert (self.held if in_place else self.held_out).tolist() == held and (self.n_free if in_place else self.n_free_out).tolist() == [left]
        if self.parents is not None:
            assert [m % 2 ** 64 for m in self.masks[:n].tolist()] == masks
        for t in (self.pos, self.slots, self.masks):
            assert bool((t[n:] == -9).all())


def requests(g, c, B, longest, most, empty, trees):
    lens = [-1 if g.random() < empty else int(g.integers(0, longest + 1)) for _ in range(B)]
    new = [int(g.integers(0, most + 1)) for _ in range(B)]
    held = [max(-(-n // 16), 0) + (int(g.integers(0, 3)) if g.random() < 0.3 else 0) for n in lens]
    width = -(-(longest + most) // 16) + 3
    tab = c.tables([16 * h for h in held], width=width)
    parents = None
    if trees:
        parents = np.full((B, most), -5, np.int32)
        for b in range(B):
            parents[b, :new[b]] = R.random_tree(g, new[b])
    return lens, new, held, tab, parents


@pytest.mark.parametrize("B,longest,most,trees", [
    (1, 0, 1, False), (1, 5000, 3000, False), (3, 40, 64, True), (64, 700, 16, True), (65, 700, 1, False), (300, 90, 33, True), (1000, 60, 70, False),
    (2, 0, 64, True), (5000, 30, 3, False), (257, 20, 5, True)])
@pytest.mark.parametrize("in_place", [False, True])
def test_plans(B, longest, most, trees, in_place):
    g = np.random.default_rng(B + most)
    c = Step((1, 1, 64), B * (-(-(longest + most) // 16) + 3), max_batch=1, seed=1)
    lens, new, held, tab, parents = requests(g, c, B, longest, most, 0.2 if B > 3 else 0.0, trees)
    p = Plan(lens, new, held, tab, c.rest, parents)
    p.run(c, in_place)
    c.c.sync(1)
    p.same(R.plan(lens, new, held, tab, c.rest, parents), in_place)
    if not in_place:   # nothing of the input has changed but the table, and its new entries are the same again
        p.run(c)
        c.c.sync(1)
        p.same(R.plan(lens, new, held, tab, c.rest, parents))
    c.c.destroy()


def test_a_plan_that_cannot_be_done_changes_nothing():
    c = Step((1, 1, 64), 40, max_batch=1, seed=2)
    lens, new, held = [17, 0, 33], [3, 16, 20], [2, 0, 3]
    tab = c.tables([16 * h for h in held], width=4)
    free = c.rest[:2]   # one for request 1 and one for request 2
    ok = Plan(lens, new, held, tab, free)
    ok.run(c)
    c.c.sync(1)
    ok.same(R.plan(lens, new, held, tab, free))
    assert ok.n_free_out.tolist() == [0]
    for name, code, kw, max_rows in [
        ("too few ids", rs.RS_ERR_NO_BLOCKS, dict(free=free[:1]), None),
        ("no id", rs.RS_ERR_NO_BLOCKS, dict(free=free[:0]), None),
        ("ids beyond the array", rs.RS_ERR_NO_BLOCKS, dict(cap=1), None),
        ("table too short", rs.RS_ERR_BAD_BLOCK, dict(new=[3, 16, 32]), None),
        ("blocks that do not hold the tokens", rs.RS_ERR_BAD_BLOCK, dict(lens=[33, 0, 33]), None),
        ("too many rows", rs.RS_ERR_BAD_ARG, {}, 38),
        ("negative length", rs.RS_ERR_BAD_ARG, dict(lens=[-2, 0, 33]), None),
        ("negative count", rs.RS_ERR_BAD_ARG, dict(new=[3, -1, 20]), None),
        ("negative blocks", rs.RS_ERR_BAD_ARG, dict(held=[2, -1, 3]), None),
        ("counts whose sum passes 32 bits", rs.RS_ERR_BAD_BLOCK, dict(new=[2 ** 31 - 1] * 3), None),
        ("more than its parents", rs.RS_ERR_BAD_ARG, dict(parents=[[-1] * 19] * 3), None),
    ]:
        for in_place in (False, True):
            a = dict(lens=lens, new=new, held=held, tab=tab, free=free)
            a.update(kw)
            rooms = dict(room=0) if name.startswith("counts") else {}
            if rooms:
                p = Plan(a["lens"], [1, 1, 1], a["held"], a["tab"], a["free"])
                p.new.copy_(i32(a["new"]))
            else:
                p = Plan(**a)
            p.run(c, in_place, max_rows=max_rows)
            with pytest.raises(rs.RapidServeError) as e:
                c.c.sync(1)
            assert e.value.code == code, name
            c.c.sync(1)
            assert p.cu.tolist() == [0] * 4, name
            assert np.array_equal(p.tab.cpu().numpy(), tab) and bool((p.pos == -9).all()) and bool((p.slots == -9).all()), name
            assert (p.held if in_place else p.held_out).tolist() == list(a["held"]), name
            assert (p.n_free if in_place else p.n_free_out).tolist() == [len(a["free"])], name
    c.c.destroy()


@pytest.mark.parametrize("B,n", [(3, 2 ** 31 - 20), (4, 2 ** 30), (70, 2 ** 26), (2000, 2 ** 22 + 1)])
def test_sums_that_pass_32_bits(B, n):
    """Counts that fit their tables (whose entries nobody reads) and whose sum is 0, small or negative in 32 bits: too many rows, nothing is done."""
    c = Step((1, 1, 64), 8, max_batch=1, seed=5)
    p = Plan([0] * B, [1] * B, [0] * B, np.full((B, 1), -1, np.int32), np.arange(8, dtype=np.int32))
    p.new.copy_(i32([n] * B))
    torch.cuda.synchronize()
    c.c.kv_plan(1, p.lens, p.new, p.held, p.tab, 2 ** 27 - 1, B, p.free, p.cap, p.n_free, 2 ** 31 - 1, p.cu, p.pos, p.slots, p.held_out, p.n_free_out)
    with pytest.raises(rs.RapidServeError) as e:
        c.c.sync(1)
    assert e.value.code == rs.RS_ERR_BAD_ARG
    assert p.cu.tolist() == [0] * (B + 1) and p.n_free_out.tolist() == [8] and bool((p.tab == -1).all()) and bool((p.pos == -9).all())
    # as many rows as the bound allows, but more blocks than there are
    p.new.copy_(i32([2 ** 31 // 4096] * B))
    torch.cuda.synchronize()
    c.c.kv_plan(1, p.lens, p.new, p.held, p.tab, 2 ** 27 - 1, B, p.free, p.cap, p.n_free, 2 ** 31 - 1, p.cu, p.pos, p.slots, p.held_out, p.n_free_out)
    with pytest.raises(rs.RapidServeError) as e:
        c.c.sync(1)
    assert e.value.code == rs.RS_ERR_NO_BLOCKS and p.cu.tolist() == [0] * (B + 1) and bool((p.tab == -1).all())
    c.c.destroy()


def test_ids_outside_the_pool_and_parents_that_come_later():
    c = Step((1, 1, 64), 40, max_batch=1, seed=3)
    free = np.array([5, 40, 7], np.int32)   # taken from the end: 7, then 40, which is none
    p = Plan([17, 10], [20, 20], [2, 1], np.array([[1, -3, -1], [2, -1, -1]], np.int32), free)
    p.run(c)
    with pytest.raises(rs.RapidServeError) as e:
        c.c.sync(1)
    assert e.value.code == rs.RS_ERR_BAD_BLOCK
    assert p.slots[:40].tolist() == [-1] * 15 + [7 * 16 + i for i in range(5)] + [2 * 16 + i for i in range(10, 16)] + [-1] * 14
    assert p.tab.tolist() == [[1, -3, 7], [2, 40, -1]]
    p = Plan([4], [4], [1], np.array([[1]], np.int32), free, parents=[[-1, 1, -2, 2]])
    p.run(c)
    with pytest.raises(rs.RapidServeError) as e:
        c.c.sync(1)
    assert e.value.code == rs.RS_ERR_BAD_ARG
    assert p.masks[:4].tolist() == [1, 2, 4, 12] and p.pos[:4].tolist() == [4, 4, 4, 5]
    c.c.destroy()


def test_plans_of_both_sides_at_once_and_recorded_ones():
    """A plan recorded in place, replayed: every replay appends to what the one before left."""
    g = np.random.default_rng(4)
    c = Step((1, 1, 64), 4000, max_batch=1, max_prefill=16, seed=4)
    B = 200
    lens, new, held, tab, _ = requests(g, c, B, 50, 6, 0.1, False)
    tab = np.pad(tab, ((0, 0), (0, 5)), constant_values=-1)
    p = Plan(lens, new, held, tab, c.rest, room=0)
    other = Plan(lens, new, held, tab, c.rest, room=0)
    stream = torch.cuda.ExternalStream(c.c.get_stream(1))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        c.c.kv_plan(1, p.lens, p.new, p.held, p.tab, tab.shape[1], B, p.free, p.cap, p.n_free, p.rows, p.cu, p.pos, p.slots, p.held, p.n_free)
    free = c.rest
    for rep in range(5):
        want = R.plan(lens, new, held, tab, free)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        other.run(c, side=0)
        c.c.sync(1), c.c.sync(0)
        p.same(want, in_place=True)
        if rep == 0:
            other.same(want)
        tab, held, free = want[0], want[5], free[:want[6]]
        lens = [a + (n if a >= 0 else 0) for a, n in zip(lens, new)]
        p.lens.copy_(i32(lens))
    del graph
    c.c.destroy()


# ---- store ----

def store(c, qkv, positions, slots, n_axes=1, pair_axis=None, n_rows=None, q="out", row_pad=8, q_pad=16, side=1, layer=0):
    n, W, Wq = len(slots), (c.Hq + 2 * c.Hkv) * c.hd, c.Hq * c.hd
    x = wide(qkv, W + row_pad)
    out = torch.full((n, Wq + q_pad), math.nan, dtype=torch.bfloat16, device="cuda")
    dp, ds = i32(positions), i32(slots)
    dn = i32([n_rows]) if n_rows is not None else None
    torch.cuda.synchronize()
    c.c.kv_store(side, layer, x, W + row_pad, {"out": out, "in place": x, None: None}[q], {"out": Wq + q_pad, "in place": W + row_pad, None: 0}[q], dp, ds, n,
                 n_rows=dn, n_axes=n_axes, pair_axis=pair_axis)
    c.c.sync(side)
    if q == "in place":
        assert torch.equal(x[:, Wq:W].cpu(), qkv.reshape(n, -1)[:, Wq:])   # keys and values stay as they were
        out = x
    elif q == "out":
        assert bool(torch.isnan(out[:, Wq:]).all())
    return out[:, :Wq].cpu().view(n, c.Hq, c.hd)


def check_store(c, qkv, positions, slots, pair_axis, got, stored, turned, layer=0):
    """Rows `turned` of the queries, rows `stored` of the cache; all else as it was."""
    Hq, Hkv, hd = c.Hq, c.Hkv, c.hd
    x = qkv.double()
    y = R.rotated(x[:, :Hq + Hkv], positions, pair_axis if pair_axis is not None else [0] * (hd // 2), c.rope_base)
    e = R.rotation_bound(x[:, :Hq + Hkv]) * (1 + 2.0 ** -8) + 2.0 ** -8 * y.abs()
    if got is not None and len(turned):
        R.held("queries", got[turned], y[turned, :Hq], e[turned, :Hq])
    k, v = c.pulled(layer)
    mine = torch.zeros(c.n_blocks * 16, dtype=torch.bool)
    s = torch.as_tensor(np.asarray(slots)[stored]).long()
    mine[s] = True
    if len(stored):
        R.held("keys", k[s // 16, s % 16], y[stored, Hq:], e[stored, Hq:])
        assert torch.equal(v[s // 16, s % 16], qkv[stored, Hq + Hkv:])
    rest = ~mine.view(c.n_blocks, 16)
    assert torch.equal(k[rest].view(torch.int16), c.k[layer][rest].view(torch.int16)) and torch.equal(v[rest].view(torch.int16), c.v[layer][rest].view(torch.int16))


AXES = {"one": (1, None), "sections": (3, lambda h: [0] * (h // 4) + [1] * (3 * h // 8) + [2] * (h - h // 4 - 3 * h // 8)),
        "interleaved": (4, lambda h: [i % 4 for i in range(h)]), "one of four": (4, lambda h: [2] * h)}


@pytest.mark.parametrize("heads", R.HEADS + [(64, 8, 128)], ids=str)
@pytest.mark.parametrize("axes", AXES)
@pytest.mark.parametrize("runs", [[(0, 1)], [(3, 50), (0, 16), (40, 9), (15, 1), (16, 33)], [(7, 8)] * 20], ids=["a token", "runs", "drafts"])
def test_store(heads, axes, runs):
    n_axes, arrange = AXES[axes]
    c = Step(heads, 60, max_batch=1, seed=5, max_pos=5000, rope_base=5e5)
    n = sum(b for _, b in runs)
    tab = c.tables([a + b for a, b in runs])
    slots = [int(tab[r, t // 16]) * 16 + t % 16 for r, (a, b) in enumerate(runs) for t in range(a, a + b)]
    positions = c.g.integers(0, 5000, (n_axes, n))
    positions[0, 0], positions[-1, -1] = 0, 4999
    pair_axis = arrange(c.hd // 2) if arrange else None
    qkv = R.bf16(c.g.standard_normal((n, c.Hq + 2 * c.Hkv, c.hd)))
    got = store(c, qkv, positions, slots, n_axes, pair_axis)
    check_store(c, qkv, positions, slots, pair_axis, got, list(range(n)), list(range(n)))
    c.c.destroy()


@pytest.mark.parametrize("heads", [(8, 2, 128), (9, 3, 128), (4, 4, 64)], ids=str)
@pytest.mark.parametrize("q", ["in place", None])
def test_store_of_shuffled_rows_with_gaps(heads, q):
    """Rows in any order, one in four without a slot, queries in place or not wanted; rows behind the last are left alone."""
    c = Step(heads, 40, max_batch=1, seed=6, max_pos=2000)
    n, rows = 300, 271
    slots = c.g.permutation(c.n_blocks * 16)[:n].astype(np.int64)
    slots[::4] = -1
    positions = c.g.integers(0, 2000, (1, n))
    qkv = R.bf16(c.g.standard_normal((n, c.Hq + 2 * c.Hkv, c.hd)))
    got = store(c, qkv, positions, slots, n_rows=rows, q=q)
    check_store(c, qkv, positions, slots, None, got if q else None, [i for i in range(rows) if i % 4], list(range(rows)))
    if q:
        assert torch.equal(got[rows:], qkv[rows:, :c.Hq])
    c.c.destroy()


@pytest.mark.parametrize("heads", [(8, 2, 128), (9, 3, 128), (4, 4, 64)], ids=str)
def test_store_of_many_rows(heads):
    """More than 2048 rows go past the caches: prompts, one behind a cached prefix that ends inside a block, rows without a slot, queries in place."""
    runs = [(5, 1200), (0, 999), (16, 33)]
    c = Step(heads, 160, max_batch=1, seed=12, max_pos=3000)
    tab = c.tables([a + b for a, b in runs])
    slots = np.array([int(tab[r, t // 16]) * 16 + t % 16 for r, (a, b) in enumerate(runs) for t in range(a, a + b)])
    slots[1500:1530] = -1
    n = len(slots)
    positions = c.g.integers(0, 3000, (2, n))
    pair_axis = [i // 3 % 2 for i in range(c.hd // 2)]
    qkv = R.bf16(c.g.standard_normal((n, c.Hq + 2 * c.Hkv, c.hd)))
    got = store(c, qkv, positions, slots, 2, pair_axis, q="in place")
    check_store(c, qkv, positions, slots, pair_axis, got, [i for i in range(n) if slots[i] >= 0], list(range(n)))
    c.c.destroy()


def test_store_skips_bad_rows_and_reports_them():
    c = Step((8, 2, 128), 10, max_batch=1, seed=7, max_pos=100)
    n = 20
    slots = list(range(32, 32 + n))
    qkv = R.bf16(c.g.standard_normal((n, 12, 128)))
    for name, bad_slot, bad_pos in (("slot", {4: 160, 9: -2, 16: 2 ** 31 - 1}, {}), ("position", {}, {0: 100, 7: -1, 19: 2 ** 31 - 1}), ("rows", {}, {})):
        s, p = list(slots), c.g.integers(0, 100, (2, n))
        for i, x in bad_slot.items():
            s[i] = x
        for i, x in bad_pos.items():
            p[i % 2, i] = x
        W = 12 * 128
        x, out = wide(qkv, W), torch.full((n, 1024), math.nan, dtype=torch.bfloat16, device="cuda")
        dp, ds, dn = i32(p), i32(s), i32([0 if name == "rows" else n])
        torch.cuda.synchronize()
        c.c.kv_store(1, 0, x, W, out, 1024, dp, ds, n, n_rows=dn, n_axes=2, pair_axis=[0, 1] * 32)
        if name == "rows":
            c.c.sync(1)
            assert bool(torch.isnan(out).all())
            continue
        with pytest.raises(rs.RapidServeError) as e:
            c.c.sync(1)
        assert e.value.code == rs.RS_ERR_BAD_BLOCK
        got = out.cpu().view(n, 8, 128)
        turned = [i for i in range(n) if i not in bad_pos]
        assert bool(torch.isnan(got[sorted(bad_pos)]).all())
        safe = np.clip(p, 0, 99)
        check_store(c, qkv, safe, s, [0, 1] * 32, got, [i for i in turned if i not in bad_slot], turned)
        c.push()
    c.c.destroy()


# ---- compact ----

def compacted(k, v, tab, ctx, keep):
    k, v = k.clone(), v.clone()
    for r, kept in enumerate(keep):
        for i, t in enumerate(kept):   # ascending, so in order
            a, b = ctx[r] + t, ctx[r] + i
            k[:, tab[r, b // 16], b % 16] = k[:, tab[r, a // 16], a % 16]
            v[:, tab[r, b // 16], b % 16] = v[:, tab[r, a // 16], a % 16]
    return k, v


@pytest.mark.parametrize("heads", R.HEADS, ids=str)
@pytest.mark.parametrize("stride", [1, 7, 64])
def test_compact(heads, stride):
    c = Step(heads, 120, max_batch=1, n_layers=3, seed=8)
    ctx = [0, 15, 16, -1, 33, 100, 47, 60, 1]
    n = len(ctx)
    tab = c.tables([max(x, 0) + 64 for x in ctx])
    keep = [sorted(c.g.choice(64, int(c.g.integers(0, stride + 1)), replace=False).tolist()) for _ in ctx]
    keep[0], keep[1] = [0][:stride], list(range(64 - stride, 64))
    dk = np.full((n, stride), -4, np.int32)
    for r, x in enumerate(keep):
        dk[r, :len(x)] = x
    keep[3] = []
    lens = [len(x) for x in keep]
    lens[3] = 5   # of a row without a request
    args = [i32(ctx), i32(dk), i32(lens), torch.from_numpy(tab).cuda()]
    torch.cuda.synchronize()
    c.c.kv_compact(1, 1, 2, args[0], args[1], stride, args[2], args[3], tab.shape[1], n)
    c.c.sync(1)
    k, v = compacted(c.k[1:], c.v[1:], tab, ctx, keep)
    for layer, (wk, wv) in enumerate([(c.k[0], c.v[0])] + list(zip(k, v))):
        gk, gv = c.pulled(layer)
        assert torch.equal(gk, wk) and torch.equal(gv, wv), layer
    c.c.destroy()


def test_compact_leaves_bad_requests_alone():
    c = Step((8, 2, 128), 40, max_batch=1, n_layers=2, seed=9)
    ctx = [10, 20, 30, -3, 40, 0, 5, 2 ** 31 - 5]
    tab = c.tables([x + 30 if 0 <= x < 100 else 30 for x in ctx])
    bad = tab.copy()
    bad[4, (40 + 9) // 16] = c.n_blocks
    keep = [[2, 2, 5], [3, 1, 4], [0, 5, 64], [1, 2, 3], [1, 9, 10], [0, 3, 9], [-1, 0, 1], [1, 2, 3]]
    for lens, code in (([3] * 8, None), ([3, 3, 3, 3, -1, 3, 4, 0], rs.RS_ERR_BAD_ARG)):
        c.push()
        args = [i32(ctx), i32(keep), i32(lens), torch.from_numpy(bad).cuda()]
        torch.cuda.synchronize()
        c.c.kv_compact(1, 0, 2, args[0], args[1], 3, args[2], args[3], tab.shape[1], 8)
        with pytest.raises(rs.RapidServeError) as e:
            c.c.sync(1)
        assert e.value.code == rs.RS_ERR_BAD_ARG
        c.c.sync(1)
        wk, wv = compacted(c.k, c.v, tab, ctx, [[], [], [], [], [], keep[5], [], []])
        for layer in range(2):
            gk, gv = c.pulled(layer)
            assert torch.equal(gk, wk[layer]) and torch.equal(gv, wv[layer])
    # a table too short, or a block that is none, alone
    for r, t in ((4, bad), (7, tab)):
        c.push()
        args = [i32(ctx[r:r + 1]), i32([[1, 9, 10]]), i32([3]), torch.from_numpy(t[r:r + 1].copy()).cuda()]
        torch.cuda.synchronize()
        c.c.kv_compact(1, 0, 2, args[0], args[1], 3, args[2], args[3], tab.shape[1], 1)
        with pytest.raises(rs.RapidServeError) as e:
            c.c.sync(1)
        assert e.value.code == rs.RS_ERR_BAD_BLOCK
        gk, gv = c.pulled(0)
        assert torch.equal(gk, c.k[0]) and torch.equal(gv, c.v[0])
    c.c.destroy()
