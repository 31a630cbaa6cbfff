"""The 4-bit cache on the GPU against its definition in float64: bytes written, rows read back, attention of both kinds."""
import numpy as np
import pytest
import torch

import paper_2601_11822_amd as rs
from tests import kv4_ref as R
from tests.gpu_util import to_bits, to_dev

pytestmark = pytest.mark.gpu

HEADS = [(4, 4, 64), (8, 2, 128), (9, 3, 128), (16, 1, 64), (32, 2, 128)]
ALL_BAD = 0xFF   # unwritten bytes: scales that read as NaN


class Cache:
    """A 4-bit context with its pool on the GPU and the same pool by the definition on the host."""

    def __init__(self, heads, n_blocks, max_prefill=0, max_batch=0, max_context=4096, n_layers=1, seed=0, fill=ALL_BAD):
        self.Hq, self.Hkv, self.hd = heads
        self.n_blocks, self.n_layers = n_blocks, n_layers
        self.g = np.random.default_rng(seed)
        self.ref = np.full((n_layers, n_blocks, self.Hkv, 17 * self.hd), fill, np.uint8)
        self.pool = torch.from_numpy(self.ref.copy()).cuda()
        self.c = rs.Context(d_model=256, n_q_heads=self.Hq, n_kv_heads=self.Hkv, head_dim=self.hd, ffn_dim=256, n_layers=n_layers, rms_eps=1e-5,
                            rope_base=1e4, max_pos=64, n_blocks=n_blocks, kv4_pool=self.pool, max_prefill_tokens=max_prefill,
                            max_decode_batch=max_batch, max_context=max_context)
        self.loud = np.exp(0.7 * self.g.standard_normal((self.Hkv, self.hd)))

    def tables(self, counts, extra=1):
        """Shuffled, disjoint blocks for each request (-1 behind them)."""
        need = [-(-n // 16) for n in counts]
        width = max(need) + extra
        perm, at = self.g.permutation(self.n_blocks), 0
        tab = np.full((len(counts), width), -1, np.int32)
        for r, n in enumerate(need):
            tab[r, :n] = perm[at:at + n]
            at += n
        assert at <= self.n_blocks
        return tab, torch.from_numpy(tab).cuda()

    def rows(self, n, loud=True):
        x = self.g.standard_normal((n, self.Hkv, self.hd)) * (self.loud if loud else 1.0)
        return R.to_bf16_bits(x.astype(np.float32))

    def fill(self, tab, counts, layer=0):
        """Puts random keys and values behind the tables, by the definition, into both pools."""
        for r, n in enumerate(counts):
            k, v = self.rows(n), self.rows(n, False)
            for t in range(n):
                R.put(self.ref[layer], self.hd, tab[r, t // 16], t % 16, R.f64(k[t]), R.f64(v[t]))
        self.pool.copy_(torch.from_numpy(self.ref))
        torch.cuda.synchronize()

    def queries(self, n):
        x = self.g.standard_normal((n, self.Hkv, self.Hq // self.Hkv, self.hd)) * 1.5 / self.loud[:, None]
        return R.to_bf16_bits(x.astype(np.float32)).reshape(n, self.Hq, self.hd)

    def same_pool(self):
        torch.cuda.synchronize()
        got = self.pool.cpu().numpy()
        assert np.array_equal(got, self.ref), f"{np.argwhere(got != self.ref)[:4]} of {got.shape}"


def wide(bits, width, stride, seed=9):
    """Rows [n, width] in a matrix of `stride` columns whose others hold NaN; returns (matrix, view's first element's tensor)."""
    m = np.full((bits.shape[0], stride), 0x7FC1, np.uint16)
    m[:, :width] = bits.reshape(bits.shape[0], width)
    return to_dev(m)


def i32(a):
    return torch.tensor(np.asarray(a, np.int32), dtype=torch.int32, device="cuda")


def put_run(cache, tab, r, start, k, v, layer=0):
    for i in range(k.shape[0]):
        t = start + i
        R.put(cache.ref[layer], cache.hd, tab[r, t // 16], t % 16, R.f64(k[i]), R.f64(v[i]))


@pytest.mark.parametrize("heads", HEADS[:4])
def test_write_append_and_read(heads):
    """Runs that start and end anywhere, an empty one, strided rows; then a token each; the bytes are the definition's, all others
    stay, and what is read back is what the bytes stand for."""
    lens, starts = [1, 0, 16, 37, 70], [5, 3, 16, 9, 0]
    held = [s + n for s, n in zip(starts, lens)]
    c = Cache(heads, 24, max_prefill=1, max_batch=8, n_layers=2)
    tab, dtab = c.tables([n + 1 for n in held])
    W = c.Hkv * c.hd
    cu = np.concatenate([[0], np.cumsum(lens)])
    k, v = c.rows(cu[-1]), c.rows(cu[-1], False)
    dk, dv = wide(k, W, W + 24), wide(v, W, W + 24)
    torch.cuda.synchronize()
    c.c.kv4_write(0, 1, dk, dv, W + 24, cu, starts, dtab, tab.shape[1])
    c.c.sync(0)
    for r in range(len(lens)):
        put_run(c, tab, r, starts[r], k[cu[r]:cu[r + 1]], v[cu[r]:cu[r + 1]], layer=1)
    c.same_pool()
    # one token each; the second request gets none
    pos = np.array(held)
    pos[1] = -1
    k1, v1 = c.rows(5), c.rows(5, False)
    dk1, dv1, dpos = wide(k1, W, W), wide(v1, W, W), i32(pos)
    torch.cuda.synchronize()
    c.c.kv4_append(1, 1, dk1, dv1, W, dpos, dtab, tab.shape[1], 5)
    c.c.sync(1)
    for r in (0, 2, 3, 4):
        put_run(c, tab, r, pos[r], k1[r:r + 1], v1[r:r + 1], layer=1)
    c.same_pool()
    # back: what was written, from the middle of a block
    lens2 = [n + 1 if r != 1 else 0 for r, n in enumerate(lens)]
    cu2 = np.concatenate([[0], np.cumsum(lens2)])
    ko, vo = (torch.full((int(cu2[-1]) + 1, W + 8), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    torch.cuda.synchronize()
    c.c.kv4_read(1, 1, ko, vo, W + 8, cu2, starts, dtab, tab.shape[1])
    c.c.sync(1)
    for r in range(5):
        want = [R.get(c.ref[1], c.hd, tab[r, t // 16], t % 16) for t in range(starts[r], starts[r] + lens2[r])]
        for o, which in ((ko, 0), (vo, 1)):
            got = R.f64(to_bits(o[cu2[r]:cu2[r + 1], :W])).reshape(-1, c.Hkv, c.hd)
            if lens2[r]:
                assert np.array_equal(got, np.array([w[which] for w in want]))
    for o in (ko, vo):
        assert (o[:, W:] == 7).all() and (o[-1] == 7).all()
    c.c.destroy()


def test_every_bf16_pattern_is_rounded_as_defined():
    """All 65536 patterns as elements: of groups of neighbours, and in front of a largest element that makes them small, tied and
    clamped; among them subnormals, infinities and NaN (whose group's codes do not matter)."""
    c = Cache((4, 4, 64), 300)
    bits = np.arange(65536, dtype=np.uint32).astype(np.uint16).reshape(-1, 4, 64)    # 256 tokens
    mixed = np.random.default_rng(3).permutation(65536).astype(np.uint16).reshape(-1, 4, 64)
    mixed = np.where((mixed & 0x7F80) == 0x7F80, mixed & 0x3FFF, mixed)
    near = (mixed & 0x81FF) | 0x3E00   # exponents of 2^-3 to 1: ties and small codes
    k, v = np.concatenate([bits, mixed]), np.concatenate([near, bits])
    tab, dtab = c.tables([512])
    dk, dv = to_dev(k.reshape(512, -1)), to_dev(v.reshape(512, -1))
    torch.cuda.synchronize()
    c.c.kv4_write(0, 0, dk, dv, 256, [0, 512], None, dtab, tab.shape[1])
    c.c.sync(0)
    put_run(c, tab, 0, 0, k, v)
    got = c.pool.cpu().numpy()
    for t in range(512):
        for a, b in zip(R.get(got[0], 64, tab[0, t // 16], t % 16), R.get(c.ref[0], 64, tab[0, t // 16], t % 16)):
            assert np.array_equal(a, b, equal_nan=True), t
    c.c.destroy()


def run_decode(c, q, ctx, dtab, width, max_ctx, stride=0, layer=0):
    W, B = c.Hq * c.hd, len(ctx)
    dq = wide(q, W, W + stride)
    out = torch.full((B + 1, W + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    dctx = i32(ctx)
    torch.cuda.synchronize()
    c.c.kv4_decode_attention(layer, dq, W + stride, out, W + 16, dctx, dtab, width, B, max_ctx)
    c.c.sync(1)
    assert (out[B] == 7).all() and (out[:, W:] == 7).all()
    return R.f64(to_bits(out[:B, :W])).reshape(B, c.Hq, c.hd)


def held_to(got, want, bound, name):
    worst = float(np.max(np.abs(got - want) / np.maximum(bound, 1e-30))) if got.size else 0.0
    print(f"  {name}: {worst:.3f} of the bound", flush=True)
    fine = bool(np.isfinite(got).all() and worst <= 1.0)
    assert fine, name


@pytest.mark.parametrize("heads", HEADS)
def test_decode_attention(heads):
    """Contexts at every border of blocks, waves and chunks, an empty row among them, over a pool whose other bytes read as NaN."""
    ctx = [0, -1, 1, 14, 15, 16, 30, 31, 32, 33, 63, 127, 128, 159, 255, 256, 511, 512, 700]
    c = Cache(heads, 260, max_batch=len(ctx), max_context=4096)
    tab, dtab = c.tables([n + 1 for n in ctx])
    c.fill(tab, [n + 1 for n in ctx])
    q = c.queries(len(ctx))
    for max_ctx in (701, min(16 * tab.shape[1], 4096)):   # two ways of cutting, or one
        got = run_decode(c, q, ctx, dtab, tab.shape[1], max_ctx, stride=8)
        for r, n in enumerate(ctx):
            k, v = R.gather(c.ref[0], c.hd, tab[r], n + 1)
            want, bound = R.attention(R.f64(q[r:r + 1]), k, v, n)
            if n < 0:
                assert (got[r] == 0).all()
            else:
                held_to(got[r:r + 1], want, bound, f"ctx {n}, max {max_ctx}")
    c.c.destroy()


@pytest.mark.parametrize("batch", [1, 2, 40, 130])
def test_decode_attention_is_the_same_however_it_is_cut(batch):
    """Long and short contexts in batches that are cut into chunks of different lengths."""
    c = Cache((8, 2, 128), 1200, max_batch=batch, max_context=9000, seed=batch)
    ctx = [int(x) for x in np.linspace(2900, 40, batch)] if batch < 40 else [int(x) for x in np.linspace(200, 1, batch)]
    tab, dtab = c.tables([n + 1 for n in ctx])
    c.fill(tab, [n + 1 for n in ctx])
    q = c.queries(batch)
    got = run_decode(c, q, ctx, dtab, tab.shape[1], max(ctx) + 1)
    for r in sorted({0, batch // 2, batch - 1}):
        k, v = R.gather(c.ref[0], c.hd, tab[r], ctx[r] + 1)
        want, bound = R.attention(R.f64(q[r:r + 1]), k, v, ctx[r])
        held_to(got[r:r + 1], want, bound, f"row {r} of {batch}")
    c.c.destroy()


MANY = [int(x) for x in np.random.default_rng(8).integers(-1, 40, 150)]
MANY[0] = MANY[1] = MANY[149] = -1
MANY[77], MANY[80] = 4800, 600


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64), (16, 1, 128)])
@pytest.mark.parametrize("ctx", [[5000, -1, 3, 700, -1, 1300], [127, 128, 255, 256, 383, 0, 126], [-1, -1, -1], [-1] * 70 + [1500], MANY, [4999]], ids=lambda x: f"{len(x)}-{max(x)}")
def test_decode_attention_in_equal_shares(heads, ctx):
    """A bound on the contexts that lets whole rows be cut anywhere: rows that are a share, a part of one and several, empty ones in
    front, between and behind, more rows than a wave has lanes."""
    c = Cache(heads, 700, max_batch=len(ctx), max_context=9000, seed=len(ctx))
    tab, _ = c.tables([n + 1 for n in ctx])
    tab = np.concatenate([tab, np.full((len(ctx), 563 - tab.shape[1]), -1, np.int32)], 1)
    dtab = torch.from_numpy(tab).cuda()
    c.fill(tab, [n + 1 for n in ctx])
    q = c.queries(len(ctx))
    got = run_decode(c, q, ctx, dtab, tab.shape[1], 9000)
    assert np.array_equal(run_decode(c, q, ctx, dtab, tab.shape[1], 9000), got)
    for r, n in enumerate(ctx):
        if n < 0:
            assert (got[r] == 0).all()
            continue
        k, v = R.gather(c.ref[0], c.hd, tab[r], n + 1)
        want, bound = R.attention(R.f64(q[r:r + 1]), k, v, n)
        held_to(got[r:r + 1], want, bound, f"row {r}, ctx {n}")
    c.c.destroy()


def run_prefill(c, q, cu, starts, dtab, width, stride=0, layer=0):
    W, T = c.Hq * c.hd, int(cu[-1])
    dq = wide(q, W, W + stride)
    out = torch.full((T + 1, W + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    c.c.kv4_prefill_attention(layer, dq, W + stride, out, W + 16, cu, starts, dtab, width)
    c.c.sync(0)
    assert (out[T] == 7).all() and (out[:, W:] == 7).all()
    return R.f64(to_bits(out[:T, :W])).reshape(T, c.Hq, c.hd)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("lens,starts", [([1], [0]), ([1, 0, 17, 130], [40, 9, 0, 5]), ([33, 64, 5], [0, 64, 1000]), ([300], [77]), ([2, 1], [0, 600])])
def test_prefill_attention(heads, lens, starts):
    held = [s + n for s, n in zip(starts, lens)]
    c = Cache(heads, 120, max_prefill=sum(lens))
    tab, dtab = c.tables(held)
    c.fill(tab, held)
    cu = np.concatenate([[0], np.cumsum(lens)])
    q = c.queries(int(cu[-1]))
    got = run_prefill(c, q, cu, starts, dtab, tab.shape[1], stride=16)
    for r, n in enumerate(lens):
        if n == 0:
            continue
        k, v = R.gather(c.ref[0], c.hd, tab[r], held[r])
        some = np.arange(n) if n <= 64 else np.unique(np.concatenate([np.arange(0, n, 7), [n - 1, n - 2]]))
        for i in some:
            want, bound = R.attention(R.f64(q[cu[r] + i:cu[r] + i + 1]), k, v, starts[r] + i)
            g = got[cu[r] + i:cu[r] + i + 1]
            fine = bool(np.isfinite(g).all() and (np.abs(g - want) <= bound).all())
            assert fine, (r, i, float(np.max(np.abs(g - want) / bound)))
    c.c.destroy()


@pytest.mark.parametrize("spoilt", [False, True])
def test_prefill_attention_of_many_rows(spoilt):
    """Enough rows for workgroups of eight waves: three requests, the columns of each of which end inside a workgroup; a key and a
    value that are not finite make the rows behind them NaN in their kv head and no others."""
    heads, lens, starts = (128, 8, 128), [2041, 1, 130], [0, 70, 333]
    held = [s + n for s, n in zip(starts, lens)]
    c = Cache(heads, 200, max_prefill=sum(lens), seed=5)
    tab, dtab = c.tables(held)
    c.fill(tab, held)
    bad_k, bad_v = 1500, 1723   # of request 0, in kv heads 1 and 6
    there = c.ref.copy()
    if spoilt:
        for pos, head, which in ((bad_k, 1, 2), (bad_v, 6, 3)):
            for g in (1, 3):   # of the dims' groups two
                there[0, tab[0, pos // 16], head, R.places(128, pos % 16)[which][g]] = 255
        c.pool.copy_(torch.from_numpy(there))
    cu = np.concatenate([[0], np.cumsum(lens)])
    q = c.queries(int(cu[-1]))
    got = run_prefill(c, q, cu, starts, dtab, tab.shape[1])
    head = np.arange(128) // 16
    nan = np.zeros((int(cu[-1]), 128), bool)
    if spoilt:
        pos = np.arange(lens[0])[:, None]
        nan[:lens[0]] = ((head == 1) & (pos >= bad_k)) | ((head == 6) & (pos >= bad_v))
    assert np.array_equal(np.isnan(got).all(-1), nan) and np.array_equal(np.isnan(got).any(-1), nan)
    some = {0: [0, 1, 15, 16, 63, 64, 500, 1023, 1024, 1499, 1500, 1700, 1722, 1723, 2039, 2040], 1: [0], 2: [0, 17, 128, 129]}
    for r, rows in some.items():
        k, v = R.gather(c.ref[0], c.hd, tab[r], held[r])
        for i in rows:
            want, bound = R.attention(R.f64(q[cu[r] + i:cu[r] + i + 1]), k, v, starts[r] + i)
            ok = ~nan[cu[r] + i]
            g = got[cu[r] + i:cu[r] + i + 1]
            fine = bool((np.abs(g - want) <= bound)[:, ok].all())
            assert fine, (r, i, float(np.max((np.abs(g - want) / bound)[:, ok])))
    c.c.destroy()


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64)])
def test_what_is_not_finite_reaches_the_rows_that_see_it_only(heads):
    """A NaN in a key, an infinity in a value: the rows in front of them are as they were, to the bit; the rows behind are NaN in
    the heads that share that kv head and as they were in the others."""
    n, bad_k, bad_v = 150, 100, 120
    c = Cache(heads, 40, max_prefill=n, max_batch=4)
    tab, dtab = c.tables([n])
    k, v = c.rows(n), c.rows(n, False)
    q = c.queries(n)
    W = c.Hkv * c.hd
    outs = []
    for spoil in (False, True):
        if spoil:
            k[bad_k, 1, 3], v[bad_v, 0, c.hd - 1] = 0x7FC0, 0xFF80
        dk, dv = to_dev(k.reshape(n, W)), to_dev(v.reshape(n, W))
        torch.cuda.synchronize()
        c.c.kv4_write(0, 0, dk, dv, W, [0, n], None, dtab, tab.shape[1])
        c.c.sync(0)
        outs.append(run_prefill(c, q, [0, n], None, dtab, tab.shape[1]))
        same_rows = torch.from_numpy(np.repeat(tab, 4, 0)).cuda()
        outs.append(run_decode(c, q[[99, 100, 119, 120]], [99, 100, 119, 120], same_rows, tab.shape[1], 150))
    clean, clean1, got, got1 = outs
    G = c.Hq // c.Hkv
    head = np.arange(c.Hq) // G
    for x, y, pos in ((clean, got, np.arange(n)), (clean1, got1, np.array([99, 100, 119, 120]))):
        nan = ((head[None, :] == 1) & (pos[:, None] >= bad_k)) | ((head[None, :] == 0) & (pos[:, None] >= bad_v))
        assert np.array_equal(y[~nan], x[~nan])
        if y is got:
            assert np.isnan(y[nan]).all()
        else:   # one row sees all of its tokens: the value's group alone is NaN there
            assert np.isnan(y[nan & (head[None, :] == 1)]).all() and np.isnan(y[nan & (head[None, :] == 0)][:, -32:]).all()
    c.c.destroy()


@pytest.mark.parametrize("bad", [0x7FC0, 0xFF80])
def test_a_query_that_is_not_finite_stays_in_its_row_and_head(bad):
    """A NaN or an infinity in one head of one row: that head of that row is NaN, everything else is as it was, to the bit; whole
    rows and shares of them, prompts uncut and cut."""
    n = 2000
    c = Cache((8, 2, 128), 300, max_prefill=40, max_batch=3, max_context=9000)
    tab, dtab = c.tables([n, n])
    c.fill(tab, [n, n])
    wide_tab = torch.from_numpy(np.concatenate([tab, np.full((2, 563 - tab.shape[1]), -1, np.int32)], 1)).cuda()
    clean = c.queries(40)
    spoilt = clean.copy()
    spoilt[1, 5, 77] = bad
    outs = []
    for q in (clean, spoilt):
        outs.append([run_decode(c, q[:2], [900, 1000], dtab, tab.shape[1], 1001), run_decode(c, q[:2], [1999, 1990], wide_tab, 563, 9000),
                     run_prefill(c, q, [0, 40, 40], None, dtab, tab.shape[1]), run_prefill(c, q[:20], [0, 20, 20], [1900, 0], dtab, tab.shape[1])])
    for x, y in zip(*outs):
        nan = np.zeros(y.shape[:2], bool)
        nan[1, 5] = True
        assert np.isnan(y[nan]).all() and np.array_equal(y[~nan], x[~nan]) and np.isfinite(x).all()
    c.c.destroy()


def test_a_prompt_of_65536_rows_of_one_head_cut_in_two():
    """More rows to join than one dimension of a launch has room for."""
    n, hd = 65536, 64
    c = Cache((1, 1, hd), n // 16, max_prefill=n, max_context=n)
    c.ref[:] = c.g.integers(0, 256, c.ref.shape, dtype=np.uint8)
    c.ref[..., 16 * hd:] = c.ref[..., 16 * hd:] % 8 + 120
    c.pool.copy_(torch.from_numpy(c.ref))
    tab, dtab = c.tables([n], extra=0)
    q = c.queries(n)
    got = run_prefill(c, q, [0, n], None, dtab, tab.shape[1])
    blocks = c.ref[0, tab[0]].reshape(1, n // 16, 17 * hd)   # a block as a head
    k, v = (np.stack(x, 1).reshape(n, 1, hd) for x in zip(*[R.get(blocks, hd, 0, t) for t in range(16)]))
    for i in (0, 1, 127, 128, 8191, 40000, n - 1):
        want, bound = R.attention(R.f64(q[i:i + 1]), k[:i + 1], v[:i + 1], i)
        held_to(got[i:i + 1], want, bound, f"row {i}")
    c.c.destroy()


def test_bad_blocks_and_lengths_are_reported_and_nothing_is_touched():
    """Ids outside the pool in every call, lengths outside the bound: nothing is read or written there, the next sync says so, and the
    other requests' results stay the same to the bit."""
    c = Cache((8, 2, 128), 64, max_prefill=100, max_batch=4)
    held = [60, 60, 60]
    tab, dtab = c.tables([64] * 3)
    c.fill(tab, held)
    W, Wq = 256, 1024
    q = c.queries(100)
    ctx = [59, 59, 59]
    good = run_decode(c, q[:3], ctx, dtab, tab.shape[1], 64)
    good_p = run_prefill(c, q[:90], [0, 30, 60, 90], [30, 30, 30], dtab, tab.shape[1])
    broken = tab.copy()
    broken[1, 1], broken[1, 3] = 64, -5
    dbad = torch.from_numpy(broken).cuda()
    rows = to_dev(c.rows(90).reshape(90, W))
    out = torch.zeros((90, Wq), dtype=torch.bfloat16, device="cuda")
    dq, dctx = to_dev(q[:90].reshape(90, Wq)), i32(ctx)
    kv = [torch.zeros((180, W), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()

    def reported(side, f, *a):
        f(*a)
        with pytest.raises(rs.RapidServeError) as e:
            c.c.sync(side)
        assert e.value.code == rs.RS_ERR_BAD_BLOCK
        c.c.sync(side)   # once

    reported(1, c.c.kv4_decode_attention, 0, dq, Wq, out, Wq, dctx, dbad, tab.shape[1], 3, 64)
    got = R.f64(to_bits(out[:3])).reshape(3, 8, 128)
    assert np.array_equal(got[[0, 2]], good[[0, 2]])
    reported(0, c.c.kv4_prefill_attention, 0, dq, Wq, out, Wq, [0, 30, 60, 90], [30, 30, 30], dbad, tab.shape[1])
    got = R.f64(to_bits(out)).reshape(90, 8, 128)
    assert np.array_equal(got[:30], good_p[:30]) and np.array_equal(got[60:], good_p[60:])
    reported(0, c.c.kv4_read, 0, 0, kv[0], kv[1], W, [0, 60, 120, 180], None, dbad, tab.shape[1])
    for which, o in enumerate(kv):
        got = R.f64(to_bits(o)).reshape(180, 2, 128)
        for r in range(3):
            for t in range(60):
                want = 0.0 if r == 1 and t // 16 in (1, 3) else R.get(c.ref[0], 128, tab[r, t // 16], t % 16)[which]
                assert (got[60 * r + t] == want).all()
    c.same_pool()
    # writes: the refused blocks' tokens go nowhere
    bits = to_bits(rows).reshape(90, 2, 128)
    reported(1, c.c.kv4_write, 1, 0, rows, rows, W, [0, 0, 60, 60], None, dbad, tab.shape[1])
    for t in list(range(16)) + list(range(32, 48)):
        R.put(c.ref[0], 128, tab[1, t // 16], t % 16, R.f64(bits[t]), R.f64(bits[t]))
    c.same_pool()
    far = i32([16 * tab.shape[1], -2, 20, 48])   # behind the table, negative, an id outside the pool twice
    four = torch.from_numpy(np.ascontiguousarray(broken[[0, 0, 1, 1]])).cuda()
    torch.cuda.synchronize()
    reported(0, c.c.kv4_append, 0, 0, rows, rows, W, far, four, tab.shape[1], 4)
    c.same_pool()
    reported(1, c.c.kv4_decode_attention, 0, dq, Wq, out, Wq, i32([59, -2, 64]), dtab, tab.shape[1], 3, 64)
    got = R.f64(to_bits(out[:3])).reshape(3, 8, 128)
    assert np.array_equal(got[0], good[0]) and (got[1] == 0).all()
    c.c.destroy()
