"""A 4-bit cache whose values say which keys counted: every token of a tile of 32 has the value 6 in one dim of the tile's own and 0 in
all others, so that a dim of the result is 6 times the weight of the few tiles that share it.  All terms of it are positive, so that the
bound on it is a small part of it, and a tile that is lost, or counted twice, is seen."""
import numpy as np

from tests import kv4_ref as R


def tile_dim(i, hd):
    return (37 * i + 11) % hd   # 37 has no factor in common with 64 or 128


def mark(pool, hd, blocks):
    """Values of a request's blocks in pool [n_blocks, heads, 17 hd] (numpy or torch, uint8), scales of 1."""
    for j, b in enumerate(blocks):
        d = tile_dim(j // 2, hd)
        v = pool[b, :, 8 * hd:16 * hd].reshape(pool.shape[1], 4, 16, hd // 32, 4)
        v[:] = 0
        v[:, :, d % 32 // 2, d // 32] = 7 << 4 * (d % 2)
        pool[b, :, 8 * hd:16 * hd] = v.reshape(pool.shape[1], 8 * hd)
        pool[b, :, 16 * hd + hd // 2:] = 127


def random_keys(g, n_blocks, heads, hd):
    """A pool [n_blocks, heads, 17 hd] of random keys of rms 0.7 and no values."""
    pool = np.zeros((n_blocks, heads, 17 * hd), np.uint8)
    pool[..., :8 * hd] = g.integers(0, 256, (n_blocks, heads, 8 * hd), dtype=np.uint8)
    pool[..., 16 * hd:16 * hd + hd // 2] = 125
    return pool


def held(pool, hd, table, n):
    """Keys and values [n, heads, hd] in float64, block by block."""
    nb, heads = -(-n // 16), pool.shape[1]
    blocks = pool[table[:nb]].reshape(1, nb * heads, 17 * hd)   # a (block, head) as a head
    both = zip(*[R.get(blocks, hd, 0, t) for t in range(16)])
    return [np.stack(x, 1).reshape(nb, heads, 16, hd).transpose(0, 2, 1, 3).reshape(nb * 16, heads, hd)[:n] for x in both]


# float32 holds no weights below 2^-126 of the largest, and of those above 2^-100 every one
TINY = 6 * 2.0 ** -100


def worst(got, want, bound):
    return float(np.max(np.abs(got - want) / np.maximum(bound, TINY)))


def steep_keys(g, n, hd):
    """Keys [n, 4, hd] whose products with a query of ones, over sqrt(hd), are by head: rising from -6 sqrt(hd) to 6 sqrt(hd) (from 2^-98 to
    2^98 at hd 128), falling likewise, near 0 but for the last token's, and in tiles of 32 that jump between the two ends."""
    ramp = np.linspace(-6, 6, n)
    a = np.zeros((n, 4))
    a[:, 0], a[:, 1], a[-1, 2] = ramp, -ramp, 6
    a[:, 3] = 6 * np.sin(2.4 * (np.arange(n) // 32))
    return R.rounded(a[..., None] + 0.3 * g.standard_normal((n, 4, hd)))


def fine_queries(g, rows, heads, hd):
    """Queries [rows, heads, hd] of which dim 0 is 1024 and dim 5 a small number that the scores depend on: against a key of 6 in dim 5 and
    another of 0 the weights tell it to 1/16 if all the bits that the bound asks for were kept, and not if the last of three terms was lost."""
    q = np.zeros((rows, heads, hd), np.float32)
    q[..., 0] = 1024
    q[..., 5] = g.uniform(-2, 2, (rows, heads))
    return R.to_bf16_bits(q)
