"""Windowed and tree attention over pools that hold NaN or infinities where no row of a launch looks: the same bits as over zeros there, in every
form (tests/host_masked_check.hip holds which sizes take which)."""
import math

import numpy as np
import pytest
import torch

import paper_2601_11822_amd as rs
from tests import test_gpu_trees as T
from tests import test_gpu_windows as W
from tests import step_ref as R
from tests.step_ref import Step

pytestmark = pytest.mark.gpu
POISON = [math.nan, math.inf, -math.inf]


def tables(c, counts, width=None):
    """As Step.tables, but block 0 is in none."""
    tab = c.tables(counts, width=width)
    tab[tab == 0] = c.rest[c.rest != 0][0]
    return tab


# (heads, positions of the rows, window, sinks, max_ctx): eight waves a row, alone and in pieces, and four; numbers of blocks, and of steps, of any parity
DECODE = [
    ((8, 2, 128), list(range(7, 160, 9)) + [-1], 70, 5, None),
    ((4, 4, 64), list(range(0, 160, 11)), 2 ** 31 - 1, 0, None),
    ((8, 2, 128), [900], 700, 4, 4096),
    ((16, 1, 64), [1003, 1020, 17], 900, 20, 8192),
    ((32, 8, 128), [11 * i % 300 for i in range(40)], 100, 33, None),
    ((16, 16, 64), [11 * i % 300 for i in range(20)], 64, 1, None),
]
# (heads, rows, positions of the first, window, sinks)
PROMPTS = [
    ((9, 3, 128), [37, 0, 1, 20], [5, 9, 0, 100], 50, 20),             # units of 32 columns
    ((32, 8, 128), [300], [16], 40, 5),
    ((32, 8, 128), [100], [3000], 3000, 5),                            # two teams, in pieces
    ((64, 16, 64), [160], [3001], 2 ** 31 - 1, 0),
    ((32, 8, 128), [1300, 100], [0, 20], 1250, 16),                    # two teams
    ((64, 16, 64), [700, 0, 300, 33, 1, 290], [0, 7, 16, 31, 200, 5], 129, 16),   # one team
    ((32, 8, 128), [2048], [5], 512, 3),
]
# (heads, cached tokens, drafted tokens, max_ctx)
TREES = [
    ((8, 2, 128), [1, 100, 130, 255], [3, 8, 0, 5], None),             # units of 32 columns
    ((32, 8, 128), [900], [8], 2056),
    ((32, 8, 128), [40 * i for i in range(40)], [1 + i % 7 for i in range(40)], None),
    ((32, 8, 128), [700, 3, 150, 31], [32, 30, 7, 32], 4032),          # two teams, in pieces
    ((64, 16, 64), [700], [63], 41064),
    ((32, 8, 128), [17 * i for i in range(32)], [32 - i % 3 for i in range(32)], 4128),   # two teams
    ((64, 4, 64), [30 * i for i in range(20)], [64 - i for i in range(20)], 9600),        # one team
    ((32, 8, 128), [100 + 7 * i for i in range(64)], [16 - i % 2 for i in range(64)], 4112),
]


def decode_case(heads, ctx, window, sinks, max_ctx):
    c = Step(heads, sum(n // 16 + 1 for n in ctx) + 3, max_batch=len(ctx), max_context=8192, seed=40)
    tab = tables(c, [n + 1 for n in ctx], max_ctx and -(-max_ctx // 16))
    q = c.queries(len(ctx))
    return c, tab, [R.window_keys(n, window, sinks) for n in ctx], lambda t: W.decode(c, t, ctx, window, sinks, q, max_ctx=max_ctx)


def prompt_case(heads, lens, starts, window, sinks):
    total = [s + n for s, n in zip(starts, lens)]
    c = Step(heads, sum(-(-n // 16) for n in total) + 3, max_prefill=sum(lens), max_context=8192, seed=41)
    tab = tables(c, total)
    q = c.queries(sum(lens))
    seen = [[j for j in range(s + n) if n and (j > s - window or j < sinks)] for s, n in zip(starts, lens)]
    return c, tab, seen, lambda t: W.prefill(c, t, lens, starts, window, sinks, q)


def tree_case(heads, ctx, lens, max_ctx):
    total = [a + b for a, b in zip(ctx, lens)]
    c = Step(heads, sum(-(-n // 16) for n in total) + 3, max_batch=len(ctx), max_context=41064, seed=42)
    tab = tables(c, total, max_ctx and -(-max_ctx // 16))
    q = c.queries(sum(lens))
    masks = [m for n in lens for m in T.paths(c.g, n)]
    return c, tab, [range(a + b) if b else [] for a, b in zip(ctx, lens)], lambda t: T.tree(c, t, ctx, lens, masks, q, max_ctx=max_ctx)


CASES = [(decode_case, a) for a in DECODE] + [(prompt_case, a) for a in PROMPTS] + [(tree_case, a) for a in TREES]
IDS = [f"{make.__name__}{i}" for i, (make, _) in enumerate(CASES)]


def same_bits(c, hidden, call):
    """hidden [n_blocks, 16]: places that hold zeros, or else what no row may notice."""
    got = []
    for fill in [0.0] + POISON:
        c.k[0, hidden], c.v[0, hidden] = fill, fill
        c.push()
        got.append(call())
    assert bool(torch.isfinite(got[0]).all()) and float(got[0].abs().sum()) > 0
    for fill, x in zip(POISON, got[1:]):
        assert torch.equal(x, got[0]), fill


@pytest.mark.parametrize("make,args", CASES, ids=IDS)
def test_blocks_that_are_in_no_table(make, args):
    c, tab, _, call = make(*args)
    hidden = torch.ones(c.n_blocks, 16, dtype=torch.bool)
    hidden[torch.from_numpy(np.unique(tab[tab >= 0])).long()] = False
    assert bool(hidden[0].all())
    same_bits(c, hidden, lambda: call(tab))
    c.c.destroy()


class Reported:
    """A context whose synchronization has to report a bad block."""

    def __init__(self, c):
        self.c = c

    def __getattr__(self, name):
        return getattr(self.c, name)

    def sync(self, side):
        with pytest.raises(rs.RapidServeError) as e:
            self.c.sync(side)
        assert e.value.code == rs.RS_ERR_BAD_BLOCK


@pytest.mark.parametrize("make,args", CASES, ids=IDS)
def test_ids_that_are_none_of_the_pool(make, args):
    """The first and the last block that each second request sees are missing: what block 0 holds does not show in their place."""
    c, tab, seen, call = make(*args)
    for r, keys in enumerate(seen):
        if r % 2 == 0 and len(keys):
            tab[r, keys[0] // 16], tab[r, keys[-1] // 16] = -2, c.n_blocks
    c.c = Reported(c.c)
    hidden = torch.zeros(c.n_blocks, 16, dtype=torch.bool)
    hidden[0] = True
    same_bits(c, hidden, lambda: call(tab))
    c.c.destroy()


@pytest.mark.parametrize("make,args", CASES, ids=IDS)
def test_places_that_no_row_sees(make, args):
    """Behind the last token, before the oldest window and behind the sinks."""
    c, tab, seen, call = make(*args)
    hidden = torch.ones(c.n_blocks, 16, dtype=torch.bool)
    for r, keys in enumerate(seen):
        keys = np.array(list(keys), np.int64)
        hidden[torch.from_numpy(tab[r][keys // 16]).long(), torch.from_numpy(keys % 16)] = False
    same_bits(c, hidden, lambda: call(tab))
    c.c.destroy()


@pytest.mark.parametrize("args", PROMPTS, ids=[f"prompt_case{i}" for i in range(len(PROMPTS))])
def test_tokens_that_only_later_rows_see(args):
    """The last token of every prompt: rows so far before it that they share no workgroup with its own row (128 columns) are the same bits."""
    heads, lens, starts = args[:3]
    c, tab, _, call = prompt_case(*args)
    per = 128 // (heads[0] // heads[1])
    early, hidden = [], torch.zeros(c.n_blocks, 16, dtype=torch.bool)
    for r, (n, first, at) in enumerate(zip(lens, starts, np.cumsum([0] + lens))):
        if n > per:
            hidden[tab[r, (first + n - 1) // 16], (first + n - 1) % 16] = True
            early += range(at, at + n - per)
    if early:
        same_bits(c, hidden, lambda: call(tab)[early])
    c.c.destroy()
