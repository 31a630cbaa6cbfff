"""Definitions in float64 of the calls on parts of a step (windowed and tree attention, plans, rotation and writes, moves), and a bf16 context
to make them on.  A cache here is k, v [n_blocks, 16, kv heads, head_dim], in the order of the tokens."""
import math

import numpy as np
import torch

import paper_2601_11822_amd as rs

HEADS = [(4, 4, 64), (8, 2, 128), (9, 3, 128), (16, 1, 64), (32, 2, 128)]
ROWS = [0, 1, 2, 3, 8, 9, 10, 11, 4, 5, 6, 7, 12, 13, 14, 15]   # row of a block's K in the pool at which token slot t stands
FULL = (1 << 64) - 1


def bf16(x):
    return torch.as_tensor(np.asarray(x, np.float32)).bfloat16()


def pools(k, v):
    """bf16 tensors in the pools' layouts."""
    n, _, h, hd = k.shape
    kp = torch.empty(n, h, hd // 32, 4, 16, 8, dtype=torch.bfloat16, device=k.device)
    kp[..., ROWS, :] = k.view(n, 16, h, hd // 32, 4, 8).permute(0, 2, 3, 4, 1, 5)
    return kp, v.permute(0, 2, 3, 1).contiguous()


def unpool(kp, vp):
    n, h = kp.shape[:2]
    return kp[..., ROWS, :].permute(0, 4, 1, 2, 3, 5).reshape(n, 16, h, -1), vp.permute(0, 3, 1, 2)


class Step:
    """A bf16 context whose cache is random, or NaN everywhere (fill="nan"), with a copy in token order."""

    def __init__(self, heads, n_blocks, max_prefill=0, max_batch=0, max_context=4096, n_layers=1, seed=0, fill="random", max_pos=64, rope_base=1e4):
        self.Hq, self.Hkv, self.hd = heads
        self.n_blocks, self.L, self.rope_base = n_blocks, n_layers, rope_base
        self.g = np.random.default_rng(seed)
        self.loud = np.exp(0.7 * self.g.standard_normal((self.Hkv, self.hd)))
        shape = (n_layers, n_blocks, 16, self.Hkv, self.hd)
        if fill == "nan":
            self.k, self.v = (torch.full(shape, math.nan, dtype=torch.bfloat16) for _ in range(2))
        else:
            self.k, self.v = bf16(self.g.standard_normal(shape) * self.loud), bf16(self.g.standard_normal(shape))
        both = [pools(self.k[i], self.v[i]) for i in range(n_layers)]
        self.kp, self.vp = (torch.stack([b[i] for b in both]).cuda() for i in range(2))
        self.c = rs.Context(d_model=256, n_q_heads=self.Hq, n_kv_heads=self.Hkv, head_dim=self.hd, ffn_dim=256, n_layers=n_layers, rms_eps=1e-5,
                            rope_base=rope_base, max_pos=max_pos, n_blocks=n_blocks, k_pool=self.kp, v_pool=self.vp, max_prefill_tokens=max_prefill,
                            max_decode_batch=max_batch, max_context=max_context)

    def push(self):
        """The copy in token order -> the pools."""
        for i in range(self.L):
            kp, vp = pools(self.k[i], self.v[i])
            self.kp[i].copy_(kp), self.vp[i].copy_(vp)
        torch.cuda.synchronize()

    def pulled(self, layer=0):
        torch.cuda.synchronize()
        return unpool(self.kp[layer].cpu(), self.vp[layer].cpu())

    def tables(self, counts, extra=1, width=None):
        """Shuffled, disjoint blocks for each request (-1 behind them)."""
        need = [-(-n // 16) for n in counts]
        width = width or max(need) + extra
        perm, at = self.g.permutation(self.n_blocks), 0
        tab = np.full((len(counts), width), -1, np.int32)
        for r, n in enumerate(need):
            tab[r, :n] = perm[at:at + n]
            at += n
        assert at <= self.n_blocks
        self.rest = perm[at:].astype(np.int32)
        return tab

    def queries(self, n):
        x = self.g.standard_normal((n, self.Hkv, self.Hq // self.Hkv, self.hd)) * 1.5 / self.loud[:, None]
        return bf16(x).reshape(n, self.Hq, self.hd)

    def tokens(self, table, at, layer=0):
        """Keys and values [n, kv heads, hd] in float64 of a request's places `at`."""
        blk, slot = torch.as_tensor(np.asarray(table)[np.asarray(at) // 16]).long(), torch.as_tensor(np.asarray(at) % 16).long()
        return self.k[layer][blk, slot].double(), self.v[layer][blk, slot].double()


def wide(x, stride, fill=math.nan):
    """Rows [n, width] on the GPU in a matrix of `stride` columns whose others hold `fill`."""
    x = x.reshape(x.shape[0], -1)
    m = torch.full((x.shape[0], stride), fill, dtype=x.dtype)
    m[:, :x.shape[1]] = x
    return m.cuda()


def i32(a):
    return torch.tensor(np.asarray(a).astype(np.int32), dtype=torch.int32, device="cuda")


def i64(a):
    return torch.tensor(np.asarray(a, np.uint64).astype(np.int64), dtype=torch.int64, device="cuda")


def attention(q, k, v):
    """One row: q [Hq, hd] over the keys and values [n, Hkv, hd] that it sees, float64.  Returns the output and a bound of what rounding
    may do to it, element by element:

    a weight goes into the product with V as bf16 (2^-8 of itself) and into the sum as float32; its score is a sum of hd products in float32,
    each of them exact, so off by at most hd 2^-24 sum|q k|, here doubled for the order of the matrix unit's sums, and the exponent of 2
    that is taken of it by two roundings of 2^-24 of its size and of the maximum's; with a relative error of delta the weight is off in the
    numerator and in the sum, twice delta in all; exponentials (2^-22) and the sums' roundings, one a key and one for each of the pieces' rescalings,
    are within 2^-14 for up to 2^9 tiles and pieces; the result is rounded to bf16 (2^-8 of itself, and of the error in front of it)."""
    Hq, hd = q.shape
    q = q.double()
    if k.shape[0] == 0:
        return torch.zeros(Hq, hd, dtype=torch.float64), torch.zeros(Hq, hd, dtype=torch.float64)
    G = Hq // k.shape[1]
    qg = q.view(-1, G, hd)
    kk, vv = k.transpose(0, 1).contiguous(), v.transpose(0, 1).contiguous()       # [Hkv, n, hd]
    s = torch.matmul(qg, kk.transpose(1, 2).contiguous()) / math.sqrt(hd)         # [Hkv, G, n]
    p = torch.softmax(s, -1)
    size = torch.matmul(qg.abs(), kk.abs().transpose(1, 2).contiguous()) / math.sqrt(hd)
    delta = 2.0 * hd * 2.0 ** -24 * size + 2.0 ** -23 * (s.abs() + s.abs().amax(-1, keepdim=True))
    delta = delta.amax(-1, keepdim=True)
    out, mass = torch.matmul(p, vv), torch.matmul(p, vv.abs())
    e = mass * (2.0 ** -8 + 2.0 * delta + 2.0 ** -14)
    return out.view(Hq, hd), (e + 2.0 ** -8 * (out.abs() + e)).view(Hq, hd)


def window_keys(pos, window, sinks):
    """Positions that the row at `pos` sees."""
    return np.array([j for j in range(pos + 1) if j > pos - window or j < sinks], np.int64)


def tree_keys(ctx, n, mask):
    return np.array(list(range(ctx)) + [ctx + t for t in range(n) if mask >> t & 1], np.int64)


def held(name, got, want, bound):
    """got, want, bound [.., Hq, hd]: inside the bound everywhere; prints the largest share of it."""
    assert bool(torch.isfinite(got).all()), name
    worst = float(((got.double() - want).abs() / bound.clamp(min=1e-30)).max()) if got.numel() else 0.0
    print(f"  {name}: {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0, name


def plan(lens, new, held_blocks, tables, free, parents=None, max_rows=None):
    """tables (changed), cu, positions, slots, masks, held, free left; None where it cannot be done."""
    lens, new, held_blocks = [[int(x) for x in a] for a in (lens, new, held_blocks)]
    n_free, top = len(free), len(free)
    tables, cu, positions, slots, masks = tables.copy(), [0], [], [], []
    out_held = list(held_blocks)
    for b, (ctx, n) in enumerate(zip(lens, new)):
        if ctx == -1:
            cu.append(cu[-1])
            continue
        while out_held[b] * 16 < ctx + n:
            if top == 0 or out_held[b] >= tables.shape[1]:
                return None
            top -= 1
            tables[b, out_held[b]] = free[top]
            out_held[b] += 1
        paths = []
        for i in range(n):
            p = -1 if parents is None else int(parents[b][i])
            paths.append((paths[p] if p >= 0 else 0) | 1 << i)
            positions.append(ctx + (i if parents is None else bin(paths[i]).count("1") - 1))
            slots.append(int(tables[b, (ctx + i) // 16]) * 16 + (ctx + i) % 16)
        masks += paths
        cu.append(cu[-1] + n)
    return tables, cu, positions, slots, masks, out_held, top


def random_tree(g, n):
    """Parents, each less than its index or -1."""
    return [int(g.integers(-1, i)) if i and g.random() < 0.5 else i - 1 for i in range(n)]


def rotated(x, positions, pair_axis, base):
    """x [n, heads, hd] float64, positions [axes, n] -> rotated, float64."""
    hd = x.shape[-1]
    i = torch.arange(hd // 2)
    pos = torch.as_tensor(np.asarray(positions))[torch.as_tensor(pair_axis).long()].t().double()
    angle = pos * torch.tensor(base, dtype=torch.float64) ** (-2.0 * i.double() / hd)
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    a, b = x[..., :hd // 2], x[..., hd // 2:]
    return torch.cat((a * c - b * s, b * c + a * s), -1)


def rotation_bound(x):
    """cos and sin are float32 (2^-24 each), the two products and their sum are rounded to float32 (2^-24 each, three), the result to bf16
    (2^-8 of it): against |a| + |b| of the pair."""
    a, b = x[..., :x.shape[-1] // 2].abs(), x[..., x.shape[-1] // 2:].abs()
    return torch.cat((a + b, a + b), -1) * (4 * 2.0 ** -24)
