"""Stores in the forms that only many rows or many bytes lead to."""
import numpy as np
import pytest

from tests import step_ref as R
from tests.step_ref import Step
from tests.test_gpu_upkeep import check_store, store

pytestmark = pytest.mark.gpu


def rows_of(c, runs):
    tab = c.tables([a + b for a, b in runs])
    return np.array([int(tab[r, t // 16]) * 16 + t % 16 for r, (a, b) in enumerate(runs) for t in range(a, a + b)])


@pytest.mark.parametrize("heads,runs", [((32, 8, 128), [(5, 2700), (0, 1400), (16, 33)]), ((64, 4, 64), [(3, 3100), (40, 1801)])], ids=str)
@pytest.mark.parametrize("q", ["out", "in place"])
def test_rows_that_go_past_the_caches(heads, runs, q):
    """More than 80 MiB read and written: prompts, one behind a cached prefix that ends inside a block, rows without a slot."""
    c = Step(heads, sum(-(-(a + b) // 16) for a, b in runs) + 2, max_batch=1, seed=60, max_pos=4000)
    slots = rows_of(c, runs)
    slots[1500:1530] = -1
    n = len(slots)
    assert n * (c.Hq + 2 * c.Hkv) * c.hd * 4 > 80 << 20
    positions = c.g.integers(0, 4000, (2, n))
    pair_axis = [i // 3 % 2 for i in range(c.hd // 2)]
    qkv = R.bf16(c.g.standard_normal((n, c.Hq + 2 * c.Hkv, c.hd)))
    got = store(c, qkv, positions, slots, 2, pair_axis, q=q)
    check_store(c, qkv, positions, slots, pair_axis, got, [i for i in range(n) if slots[i] >= 0], list(range(n)))
    c.c.destroy()


@pytest.mark.parametrize("heads", [(8, 2, 128), (9, 3, 128), (16, 16, 64)], ids=str)
@pytest.mark.parametrize("bound,rows", [(2100, [0, 1, 61, 2047, 2048, 2049, 2100]), (9000, [3, 1900, 2050])], ids=str)
def test_fewer_rows_than_the_bound(heads, bound, rows):
    """A recorded call's bound of its rows, and the rows there are, on either side of 2048: short runs first, then a long one."""
    runs = [(7 * i % 30, 1 + i % 9) for i in range(40)]
    runs.append((2, bound - sum(b for _, b in runs)))
    c = Step(heads, sum(-(-(a + b) // 16) for a, b in runs) + 2, max_batch=1, seed=61, max_pos=9100)
    slots = rows_of(c, runs)
    positions = c.g.integers(0, 9100, (1, bound))
    qkv = R.bf16(c.g.standard_normal((bound, c.Hq + 2 * c.Hkv, c.hd)))
    for n in rows:
        got = store(c, qkv, positions, slots, n_rows=n, q="in place")
        check_store(c, qkv, positions, slots, None, got, list(range(n)), list(range(n)))
        assert bool((got[n:] == qkv[n:, :c.Hq]).all())
        c.push()
    c.c.destroy()
