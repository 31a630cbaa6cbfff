"""The operators of the 4-bit paged KV cache: calls a serving program makes of a context whose cache is held in 4 bits.

kind "store":   keys and values of new tokens are quantised into the cache (runs of tokens of several requests, or one token
                each), and every request is read back whole: what was there before and what was written.
kind "read":    whole requests read back to bf16 rows.
kind "decode":  attention of one row per request over its cached tokens.
kind "prefill": causal attention of several rows per request, the last of its cached tokens.

The cache: blocks of 16 tokens; of a (block, kv head) 17 * head_dim bytes: the codes of K [head_dim/32][16 tokens][16], where a byte
holds dims 2j (low half) and 2j+1 of a group of 32; the codes of V [4][16][head_dim/32][4], where byte (q, j, g, i) holds dims
32g+2j and 32g+2j+1 of token 4q+i; a scale byte b (2^(b-127), 255: not a number) for each token and group, those of K
[head_dim/32][16] and of V [4][head_dim/32][4].  A code is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6.

Lengths follow from the case alone, so that every seed is the same amount of work; the seed draws the values, the order of the
requests and the blocks.
"""
import math

import numpy as np
import torch

own = False

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(kind, name=None, hq=32, hkv=8, hd=128, prompts="", starts="", batch=0, ctx_lo=0, ctx_hi=0, empty=0):
    c = dict(kind=kind, hq=hq, hkv=hkv, hd=hd, prompts=prompts, starts=starts, batch=batch, ctx_lo=ctx_lo, ctx_hi=ctx_hi, empty=empty)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one user's chat turn: the step's token joins 900 cached ones (latency and the number of launches count)
        _case("store", "store_1", batch=1, ctx_lo=900, ctx_hi=900),
        # a decode batch of short contexts, a token each
        _case("store", "store_64", batch=64, ctx_lo=30, ctx_hi=500),
        # prompts of uneven lengths that were prefilled together, two of them behind cached prefixes that end inside a block
        _case("store", "store_ragged", hq=64, prompts="1391,518,2730,805", starts="0,1037,0,250"),
        # a long request's cache as bf16 rows (handed to another program)
        _case("read", "read_32768", prompts="32768"),
        # one user's chat turn
        _case("decode", "decode_1", batch=1, ctx_lo=900, ctx_hi=900),
        # the benchmark's decode batch
        _case("decode", "decode_64", batch=64, ctx_lo=512, ctx_hi=4096),
        # the long-context configuration: reading the cache is all there is
        _case("decode", "decode_long", batch=32, ctx_lo=8192, ctx_hi=32767),
        # heads of 64, many short contexts, and rows without a request that fill up a captured batch
        _case("decode", "decode_hd64", hq=32, hkv=4, hd=64, batch=203, ctx_lo=1, ctx_hi=1500, empty=53),
        # a question of few rows behind a long conversation
        _case("prefill", "prefill_19_behind", prompts="19", starts="6005"),
        # the benchmark's prompt
        _case("prefill", "prefill_2048", prompts="2048"),
        # the 70B-shaped configuration's heads: chunks of prompts behind cached ones, of uneven lengths
        _case("prefill", "prefill_ragged_70b", hq=64, prompts="700,33,1391", starts="1024,4000,0"),
        # the long-context configuration's whole prompt
        _case("prefill", "prefill_16384", prompts="16384"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(("store", "store", "read", "decode", "decode", "decode", "prefill", "prefill", "prefill"))
    hq, hkv, hd = rng.choice(((32, 8, 128), (64, 8, 128), (8, 2, 128), (32, 4, 64), (9, 3, 128), (16, 16, 64), (16, 1, 128)))
    join = lambda v: ",".join(str(x) for x in v)
    if kind == "decode" or kind == "store" and rng.random() < 0.5:
        batch = _log_uniform(rng, 1, 256 if kind == "decode" else 64)
        hi = _log_uniform(rng, 16, min(32767, max(64, (600000 if kind == "decode" else 40000) // batch)))
        return _case(kind, hq=hq, hkv=hkv, hd=hd, batch=batch, ctx_lo=rng.randint(0, hi), ctx_hi=hi,
                     empty=rng.randint(0, batch // 4) if kind == "decode" else 0)
    n = rng.randint(1, 5)
    total = _log_uniform(rng, 1, 5000 if kind == "prefill" else 16000)
    weights = [0.2 + rng.random() for _ in range(n)]
    lens = [max(1, int(total * w / sum(weights))) for w in weights]
    starts = [0 if rng.random() < 0.5 else _log_uniform(rng, 1, 6000 if kind == "prefill" else 2000) for _ in lens]
    if kind == "read":
        lens, starts = [s + m for s, m in zip(starts, lens)], []
    return _case(kind, hq=hq, hkv=hkv, hd=hd, prompts=join(lens), starts=join(starts))


def _ints(text):
    return [int(v) for v in text.split(",")] if text else []


def _lengths(case):
    """(first position, rows) of each request; of a row without a request (-1, 0)."""
    if case["batch"]:
        n = case["batch"] - case["empty"]
        return [(int(round(c)), 1) for c in np.linspace(case["ctx_lo"], case["ctx_hi"], n)] + [(-1, 0)] * case["empty"]
    lens = _ints(case["prompts"])
    return list(zip(_ints(case["starts"]) or [0] * len(lens), lens))


# ---- the plain forms -------------------------------------------------------------------------------------------------

def _quantise(x):
    """x [..., head_dim] bf16 -> codes uint8 [..., head_dim/32, 16], scale bytes uint8 [..., head_dim/32]."""
    x = x.float().unflatten(-1, (-1, 32))
    amax = x.abs().amax(-1)
    bad = ~torch.isfinite(amax)
    # the exponent field of amax, one more from 1.75 on, less 2: the largest value is less than 7 steps of 1
    b = ((torch.where(bad, 0.0, amax).view(torch.int32) + 0x200000) >> 23) - 2
    b = b.clamp(2, 252)
    y = torch.where(bad[..., None], 0.0, x) * torch.exp2(127.0 - b.double())[..., None].float()
    a = y.abs()
    # nearest level, ties to the even code
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = code + 8 * torch.signbit(y).int()
    packed = (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8)
    return packed, torch.where(bad, 255, b).to(torch.uint8)


def _parts(pool, hd):
    """Views of the pool [blocks, kv heads, 17 * head_dim]: K codes, V codes, K scales, V scales."""
    g = hd // 32
    n, h = pool.shape[:2]
    return (pool[..., :8 * hd].view(n, h, g, 16, 16), pool[..., 8 * hd:16 * hd].view(n, h, 4, 16, g, 4),
            pool[..., 16 * hd:16 * hd + hd // 2].view(n, h, g, 16), pool[..., 16 * hd + hd // 2:].view(n, h, 4, g, 4))


def _store(pool, hd, k, v, blocks, slots):
    """Quantises rows k, v [n, kv heads, head_dim] into (blocks[i], slots[i])."""
    kc, vc, ks, vs = _parts(pool, hd)
    codes, scales = _quantise(k)
    kc[blocks, :, :, slots] = codes
    ks[blocks, :, :, slots] = scales
    codes, scales = _quantise(v)
    q, i = slots // 4, slots % 4
    vc[blocks, :, q, :, :, i] = codes.transpose(-1, -2)
    vs[blocks, :, q, :, i] = scales


def _values(codes, scales):
    """Codes [..., n] of groups with one scale byte each [...] -> float32 [..., n, 2]."""
    levels = torch.tensor(LEVELS, device=codes.device)
    levels = torch.cat((levels, -levels))
    pair = torch.stack((codes & 15, codes >> 4), -1)
    s = torch.where(scales == 255, math.nan, torch.exp2(scales.double() - 127.0)).float()
    return levels.index_select(0, pair.flatten().int()).view(pair.shape) * s[..., None, None]


def _load(pool, hd, ids):
    """Blocks ids [n] -> keys and values float32 [n * 16, kv heads, head_dim]."""
    kc, vc, ks, vs = (p[ids] for p in _parts(pool, hd))
    n, h = kc.shape[:2]
    k = _values(kc, ks).permute(0, 3, 1, 2, 4, 5).reshape(n * 16, h, hd)
    v = _values(vc.transpose(3, 5).transpose(3, 4), vs).permute(0, 2, 4, 1, 3, 5, 6).reshape(n * 16, h, hd)
    return k, v


def _store_plain(st):
    hd, h = st["hd"], st["hkv"]
    if st["k"] is not None:
        _store(st["pool"], hd, st["k"].view(-1, h, hd), st["v"].view(-1, h, hd), st["blocks"], st["slots"])
    k, v = _load(st["pool"], hd, st["ids"])
    return {"k": k[st["held"]].flatten(1).bfloat16(), "v": v[st["held"]].flatten(1).bfloat16()}


def _decode_plain(st):
    B, hq, h, hd = st["B"], st["hq"], st["hkv"], st["hd"]
    k, v = _load(st["pool"], hd, st["tables"].clamp(min=0).flatten().long())
    n = k.shape[0] // B
    k, v = (x.view(B, n, h, hd).transpose(1, 2) for x in (k, v))
    q = st["q"].float().view(B, h, hq // h, hd)
    seen = torch.arange(n, device=k.device) <= st["ctx"][:, None]
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(hd)
    s = s.masked_fill(~seen[:, None, None], -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min))
    o = torch.matmul(p, v.masked_fill(~seen[:, None, :, None], 0.0)) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    return o.reshape(B, hq * hd).bfloat16()


def _prefill_plain(st):
    hq, h, hd = st["hq"], st["hkv"], st["hd"]
    q = st["q"].float().view(-1, h, hq // h, hd)
    out = torch.empty_like(st["q"]).view(-1, h, hq // h, hd)
    for r, (start, rows) in enumerate(st["lengths"]):
        at, tot = st["cu"][r], start + rows
        k, v = _load(st["pool"], hd, st["tables"][r, :-(-tot // 16)].long())
        hidden = torch.arange(tot, device=k.device) > torch.arange(start, tot, device=k.device)[:, None]
        for head in range(h):  # a kv head at a time: the scores of all at once are tens of gigabytes
            s = torch.matmul(q[at:at + rows, head].transpose(0, 1), k[:tot, head].t().contiguous()) / math.sqrt(hd)
            s = s.masked_fill(hidden, -math.inf)
            p = torch.exp(s - s.amax(-1, keepdim=True))
            out[at:at + rows, head] = (torch.matmul(p, v[:tot, head].contiguous()) / p.sum(-1, keepdim=True)).transpose(0, 1).bfloat16()
    return out.view(-1, hq * hd)


# ---- what a program holds, and its calls ---------------------------------------------------------------------------------

def prepare(case, seed):
    hq, h, hd = case["hq"], case["hkv"], case["hd"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    host = np.random.Generator(np.random.Philox(key=[seed, 0]))
    lengths = _lengths(case)
    if case["batch"]:
        lengths = [lengths[i] for i in host.permutation(len(lengths))]
    held = [s + n for s, n in lengths]
    held = [max(n, 0) for n in held]
    width = max(-(-n // 16) for n in held)
    n_blocks = sum(-(-n // 16) for n in held) + 16
    perm, at = host.permutation(n_blocks).astype(np.int32), 0
    tables = np.full((len(held), width), -1, np.int32)
    for r, n in enumerate(held):
        tables[r, :-(-n // 16)] = perm[at:at - (-n // 16)]
        at += -(-n // 16)

    # keys have a few channels much larger than the rest, as keys do
    loud = torch.exp(0.7 * torch.randn(h, hd, generator=gen, device="cuda"))
    pool = torch.empty(n_blocks, h, 17 * hd, dtype=torch.uint8, device="cuda")
    every = torch.arange(16 * n_blocks, device="cuda")
    for part in every.split(65536):
        normal = lambda: torch.randn(part.numel(), h, hd, generator=gen, device="cuda")
        _store(pool, hd, (normal() * loud).bfloat16(), normal().bfloat16(), part // 16, part % 16)

    rows = sum(n for _, n in lengths) if not case["batch"] else case["batch"]
    cu = [0]
    for _, n in lengths:
        cu.append(cu[-1] + n)
    st = dict(kind=case["kind"], hq=hq, hkv=h, hd=hd, B=case["batch"], lengths=lengths, starts=[s for s, _ in lengths], cu=cu, width=width,
              pool=pool, tables=torch.from_numpy(tables).cuda(), ctx=torch.tensor([s for s, _ in lengths], dtype=torch.int32, device="cuda"),
              max_ctx=max(held), max_held=max(held))
    if case["kind"] in ("store", "read"):
        total = sum(held)
        st["held_cu"] = [0] + [int(x) for x in np.cumsum(held)]
        # where in the blocks of all tables the requests' tokens are (what the plain form indexes with)
        ids = [tables[r, :-(-n // 16)] for r, n in enumerate(held)]
        first = np.cumsum([0] + [16 * len(b) for b in ids])
        st["ids"] = torch.from_numpy(np.concatenate(ids)).cuda().long()
        st["held"] = torch.from_numpy(np.concatenate([first[r] + np.arange(n) for r, n in enumerate(held)])).cuda()
        pos = np.concatenate([s + np.arange(n) for s, n in lengths])
        req = np.repeat(np.arange(len(lengths)), [n for _, n in lengths])
        st["blocks"], st["slots"] = torch.from_numpy(tables[req, pos // 16]).cuda().long(), torch.from_numpy(pos % 16).cuda()
        st["k_out"], st["v_out"] = (torch.empty(total, h * hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        st["k"] = st["v"] = None
        if case["kind"] == "store":
            # new keys and values as they stand in a projection's output: q | k | v of each row
            qkv = torch.randn(rows, (hq + 2 * h) * hd, generator=gen, device="cuda")
            qkv[:, hq * hd:(hq + h) * hd] *= loud.flatten()
            qkv = qkv.bfloat16()
            st["row"], st["k"], st["v"] = qkv.shape[1], qkv[:, hq * hd:(hq + h) * hd], qkv[:, (hq + h) * hd:]
    else:
        st["q"] = (torch.randn(rows, h, hq // h, hd, generator=gen, device="cuda") / loud[:, None]).bfloat16().view(rows, hq * hd)
        st["out"] = torch.empty_like(st["q"])
    if own:
        _enter(case, st, max(held), rows)
    return st


class _Program:
    """What a serving program makes when it starts: one context, and the pool of its layers' caches.  Every call goes to the streams
    of that context, one behind another."""

    def __init__(self, case, pool, max_context, rows):
        import paper_2601_11822_amd as rs
        self.case = case
        self.free = list(range(4))  # layers
        self.pool = torch.empty(len(self.free), *pool.shape, dtype=torch.uint8, device="cuda")
        self.c = rs.Context(d_model=case["hq"] * case["hd"], n_q_heads=case["hq"], n_kv_heads=case["hkv"], head_dim=case["hd"],
                            ffn_dim=case["hq"] * case["hd"], n_layers=len(self.free), rms_eps=1e-5, rope_base=500000.0, max_pos=max_context,
                            n_blocks=pool.shape[0], kv4_pool=self.pool, max_prefill_tokens=0 if case["batch"] else rows,
                            max_decode_batch=case["batch"], max_context=max_context)

    def __del__(self):
        if hasattr(self, "c"):
            self.c.destroy()


class _Layer:
    """A layer of a program's cache, until nobody holds it any more."""

    def __init__(self, program):
        self.program, self.at = program, program.free.pop()

    def __del__(self):
        self.program.free.append(self.at)


def _enter(case, st, max_context, rows):
    """Puts the cache that `st` begins with into a layer of the program for the case's sizes (the one that runs, if it is for them and has
    a layer free).  Nothing that a call computes is done here: no row is quantised or laid out, no context cut; the copied bytes are those
    that the plain form reads."""
    sizes = {k: v for k, v in case.items() if k != "name"}
    program = getattr(_enter, "program", None)
    if program is None or program.case != sizes or not program.free:
        program = _enter.program = _Program(sizes, st["pool"], max_context, rows)
    torch.cuda.synchronize()  # a layer given back may still be read
    layer = _Layer(program)
    program.pool[layer.at].copy_(st["pool"])
    st["held_by"], st["c"], st["layer"], st["pool"] = layer, program.c, layer.at, program.pool[layer.at]


def _store_own(st):
    c, layer, side = st["c"], st["layer"], 1 if st["B"] else 0  # RS_SIDE_DECODE, RS_SIDE_PREFILL
    if st["k"] is not None and st["B"]:
        c.kv4_append(side, layer, st["k"], st["v"], st["row"], st["ctx"], st["tables"], st["width"], st["B"])
    elif st["k"] is not None:
        c.kv4_write(side, layer, st["k"], st["v"], st["row"], st["cu"], st["starts"], st["tables"], st["width"])
    c.kv4_read(side, layer, st["k_out"], st["v_out"], st["hkv"] * st["hd"], st["held_cu"], None, st["tables"], st["width"])
    return {"k": st["k_out"], "v": st["v_out"]}


def _decode_own(st):
    row = st["hq"] * st["hd"]
    st["c"].kv4_decode_attention(st["layer"], st["q"], row, st["out"], row, st["ctx"], st["tables"], st["width"], st["B"], st["max_ctx"])
    return st["out"]


def _prefill_own(st):
    row = st["hq"] * st["hd"]
    st["c"].kv4_prefill_attention(st["layer"], st["q"], row, st["out"], row, st["cu"], st["starts"], st["tables"], st["width"])
    return st["out"]


def run(state):
    if state["kind"] in ("store", "read"):
        return _store_own(state) if own else _store_plain(state)
    if state["kind"] == "decode":
        return _decode_own(state) if own else _decode_plain(state)
    return _prefill_own(state) if own else _prefill_plain(state)


def work(case):
    """Cached tokens that a pass uses read once (8.5 bits for each pair of elements), bf16 rows read or written once."""
    hq, h, hd = case["hq"], case["hkv"], case["hd"]
    token = h * 17 * hd // 16  # a token's keys and values
    lengths = _lengths(case)
    held, rows = sum(max(s + n, 0) for s, n in lengths), sum(n for _, n in lengths)
    if case["kind"] == "read":
        return {"bytes": float(held * (token + 4 * h * hd)), "flops": 0.0}
    if case["kind"] == "store":
        return {"bytes": float(rows * (4 * h * hd + token) + held * (token + 4 * h * hd)), "flops": 0.0}
    pairs = sum(n * s + n * (n + 1) / 2 for s, n in lengths)
    rows = max(rows, case["batch"])
    return {"bytes": float(held * token + 4 * rows * hq * hd), "flops": float(4 * hq * hd * pairs)}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------------

def _defined(byte, scale):
    """The two values of a byte of codes, float64, by the format's definition: sign, two bits of exponent, one of fraction."""
    both = torch.stack((byte % 16, byte // 16), -1).double()
    sign = 1.0 - 2.0 * (both >= 8).double()
    mag = both % 8
    e, f = torch.div(mag, 2, rounding_mode="floor"), mag % 2
    value = torch.where(e == 0, 0.5 * f, (1.0 + 0.5 * f) * 2.0 ** (e - 1.0))
    return sign * value * torch.where(scale == 255, math.nan, 2.0 ** (scale.double() - 127.0))[..., None]


def _request(pool, hd, table, tokens):
    """Keys and values [tokens, kv heads, head_dim] in float64, token by token of a request's table."""
    h, g = pool.shape[1], hd // 32
    t = torch.arange(tokens, device=pool.device)
    rows = pool[table.long()[t // 16]]  # the token's block
    slot = t % 16
    dims = torch.arange(hd // 2, device=pool.device)
    group, j = dims // 16, dims % 16
    at_k = (group * 16 + slot[:, None]) * 16 + j
    at_v = 8 * hd + (((slot[:, None] // 4) * 16 + j) * g + group) * 4 + slot[:, None] % 4
    at_ks = 16 * hd + group * 16 + slot[:, None]
    at_vs = 16 * hd + hd // 2 + ((slot[:, None] // 4) * g + group) * 4 + slot[:, None] % 4
    pick = lambda at: rows.gather(2, at[:, None, :].expand(-1, h, -1))
    return _defined(pick(at_k), pick(at_ks)).flatten(2), _defined(pick(at_v), pick(at_vs)).flatten(2)


def _rounded(x):
    """x [..., head_dim] in float64 -> what the cache holds of it: the nearest multiple of the group's scale."""
    x = x.unflatten(-1, (-1, 32))
    amax = x.abs().amax(-1, keepdim=True)
    # the smallest power of two of which 7 are more than amax
    n = torch.ceil(torch.log2(amax / 7.0)).nan_to_num(neginf=-125.0).clamp(-125, 125)
    n = torch.where(amax >= 7.0 * 2.0 ** n, n + 1, torch.where(amax < 7.0 * 2.0 ** (n - 1), n - 1, n)).clamp(-125, 125)
    y = x.abs() / 2.0 ** n
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
    y = (torch.round(y / step) * step).clamp(max=6.0)  # to the even multiple at a tie: the even code
    return (torch.sign(x) * y * 2.0 ** n).flatten(-2)


def exact(case, seed):
    st = prepare(case, seed)
    hq, h, hd = st["hq"], st["hkv"], st["hd"]
    if case["kind"] in ("store", "read"):
        keys, values = [], []
        for r, (start, rows) in enumerate(st["lengths"]):
            k, v = _request(st["pool"], hd, st["tables"][r], start + rows)
            if case["kind"] == "store":
                new = slice(st["cu"][r], st["cu"][r + 1])
                k[start:], v[start:] = _rounded(st["k"][new].double().view(-1, h, hd)), _rounded(st["v"][new].double().view(-1, h, hd))
            keys.append(k.flatten(1)), values.append(v.flatten(1))
        return {"k": torch.cat(keys), "v": torch.cat(values)}
    q = st["q"].double().view(-1, h, hq // h, hd)
    out = torch.zeros_like(q)
    for r, (start, rows) in enumerate(st["lengths"]):
        if rows == 0:
            continue
        at, tot = (r if case["batch"] else st["cu"][r]), start + rows
        k, v = _request(st["pool"], hd, st["tables"][r], tot)
        for head in range(h):
            for first in range(0, rows, 2048):
                some = slice(first, min(rows, first + 2048))
                s = torch.einsum("rgd,td->grt", q[at:at + rows, head][some], k[:, head]) / math.sqrt(hd)
                pos = start + torch.arange(some.start, some.stop, device=s.device)
                s = torch.where(torch.arange(tot, device=s.device) <= pos[:, None], s, -math.inf)
                out[at + some.start:at + some.stop, head] = torch.einsum("grt,td->rgd", torch.softmax(s, -1), v[:, head])
    return out.view(-1, hq * hd)
