"""What the bounds of the 4-bit attention tests can see: mistakes planted in the definition, on the CPU (no GPU)."""
import math

import numpy as np
import pytest

from tests import kv4_marks as M
from tests import kv4_ref as R


def test_marks_lie_where_they_are_said_to():
    g = np.random.default_rng(0)
    for hd in (64, 128):
        pool, table = M.random_keys(g, 9, 2, hd), g.permutation(9)
        M.mark(pool, hd, table[:7])
        k, v = M.held(pool, hd, table, 105)
        slow_k, slow_v = R.gather(pool, hd, table, 105)
        assert np.array_equal(k, slow_k) and np.array_equal(v, slow_v)
        for t in range(105):
            assert (v[t, :, M.tile_dim(t // 32, hd)] == 6).all() and (np.count_nonzero(v[t], axis=-1) == 1).all()
        assert 0.6 < k.std() < 0.85


@pytest.mark.parametrize("n,hd", [(700, 64), (5000, 128), (20000, 64), (30001, 128)])
def test_a_lost_tile_is_seen_at_any_length(n, hd):
    """Any tile left out or counted twice: more than twice the bound."""
    g = np.random.default_rng(n)
    pool = M.random_keys(g, -(-n // 16), 1, hd)
    M.mark(pool, hd, np.arange(pool.shape[0]))
    k, v = M.held(pool, hd, np.arange(pool.shape[0]), n)
    q = R.f64(R.to_bf16_bits((0.4 * g.standard_normal((1, 1, hd))).astype(np.float32)))
    want, bound = R.attention(q, k, v, n - 1)
    p = np.exp(k[:, 0] @ q[0, 0] / math.sqrt(hd))
    tiles = (n + 31) // 32
    for tile in [0, 1, tiles // 3, tiles // 2, tiles - 2]:
        for times in (0, 2):
            w = p.copy()
            w[32 * tile:32 * tile + 32] *= times
            assert M.worst(w @ v[:, 0] / w.sum(), want[0, 0], bound[0, 0]) > 2, (tile, times)
    assert M.worst(p @ v[:, 0] / p.sum(), want[0, 0], bound[0, 0]) < 1e-6


def in_terms(x, terms):
    """32 dims as `terms` 6-bit terms (1 sign, 2 bits of exponent, 3 of fraction), each a sixteenth of the one before."""
    unit = 2.0 ** np.floor(np.log2(np.abs(x).max() / 1.9375) - 1 + 1e-12)
    out, rest = np.zeros_like(x), x.astype(np.float64).copy()
    for i in range(terms):
        u = unit / 16 ** i
        step = np.where(np.abs(rest) / u < 2, 1 / 8, np.where(np.abs(rest) / u < 4, 1 / 4, 1 / 2)) * u
        t = np.clip(np.round(rest / step) * step, -7.5 * u, 7.5 * u)
        out += t
        rest -= t
    return out


@pytest.mark.parametrize("hd", [64, 128])
def test_lost_terms_of_the_query_are_seen(hd):
    g = np.random.default_rng(hd)
    q = R.f64(M.fine_queries(g, 64, 1, hd))
    k, v = np.zeros((2, 1, hd)), np.zeros((2, 1, hd))
    k[1, 0, 5] = 6
    v[0, 0, 0] = v[1, 0, 1] = 6
    by = {}
    for terms in (1, 2, 3):
        by[terms] = 0.0
        for r in range(64):
            want, bound = R.attention(q[r:r + 1], k, v, 1)
            x = q[r, 0].copy()
            x[:32] = in_terms(x[:32], terms)
            s = k[:, 0] @ x / math.sqrt(hd)
            p = np.exp(s - s.max())
            by[terms] = max(by[terms], M.worst(p @ v[:, 0] / p.sum(), want[0, 0], bound[0, 0]))
    print(by)
    assert by[3] < 0.6 and by[2] > 1.2 and by[1] > 3


def test_scores_that_run_over_hundreds_of_powers_of_two():
    g = np.random.default_rng(1)
    k = M.steep_keys(g, 1500, 128)
    s = k.sum(-1) / math.sqrt(128) * math.log2(math.e)
    assert s[:, 0].min() < -90 and s[:, 0].max() > 90 and s[-1, 2] > 90 and np.abs(s[:-1, 2]).max() < 10
    steps = np.diff(np.maximum.accumulate(s[:, 0].reshape(-1, 50).max(1)))
    assert (steps > 2).mean() > 0.8   # the maximum moves in nearly every tile
