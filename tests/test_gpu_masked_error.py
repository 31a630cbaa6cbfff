"""The error of windowed and tree attention in the 2-norm: two roundings to bf16 are theirs, the weights as factors of V (below 1, the largest of a
workgroup's in [1/2, 1]), and the output.  The error is no larger than that of a float64 evaluation with these two roundings (2 % for the sample, as for
the causal prompt kernel; weights relative to a reference far behind the maximum, anywhere in their binades, showed 2 to 7 % more)."""
import numpy as np
import pytest
import torch

from tests import test_gpu_trees as T
from tests import test_gpu_windows as W
from tests.step_ref import Step

pytestmark = pytest.mark.gpu
H128, H64 = (32, 8, 128), (32, 4, 64)


def squares(c, table, sees, q, got):
    """Of one request: squares of the error and of the two roundings'.  sees [rows, keys]; q, got [rows, Hq, hd]."""
    k, v = (x.cuda() for x in c.tokens(table, np.arange(sees.shape[1])))
    sees, q, got = torch.from_numpy(sees).cuda(), q.cuda().double(), got.cuda().double()
    err = ideal = 0.0
    for h in range(c.Hq):
        at = h * c.Hkv // c.Hq
        s = (q[:, h].contiguous() @ k[:, at].t().contiguous() / c.hd ** 0.5).masked_fill(~sees, float("-inf"))
        p, values = (s - s.max(1, keepdim=True).values).exp(), v[:, at].contiguous()
        total = p.sum(1, keepdim=True)
        exact, rounded = p @ values / total, (p.bfloat16().double() @ values / total).bfloat16().double()
        err += float((got[:, h] - exact).square().sum())
        ideal += float((rounded - exact).square().sum())
    return err, ideal


def held(parts):
    err, ideal = (sum(x) for x in zip(*parts))
    print(f"  error {(err / ideal) ** 0.5:.4f} of the two roundings'", flush=True)
    assert err <= 1.02 ** 2 * ideal


@pytest.mark.parametrize("heads,lens,starts,window", [
    (H128, [300], [0], 4096),                             # units of 32 columns
    (H128, [100], [3000], 2048),                          # in pieces
    (H128, [2048], [0], 4096),                            # two teams
    (H128, [512], [3000], 2048),                          # in pieces
    (H64, [1000], [500], 4096),
    (H128, [2500], [0], 4096),                            # one team
    (H128, [2048], [0], 512),
    ((64, 8, 128), [700, 33, 1391], [1024, 4000, 0], 512),
    (H64, [2500], [0], 4096),
], ids=str)
def test_prompt_rows(heads, lens, starts, window):
    total = [s + n for s, n in zip(starts, lens)]
    c = Step(heads, sum(-(-n // 16) for n in total), max_prefill=sum(lens), max_context=8192, seed=50)
    tab = c.tables(total)
    q = c.queries(sum(lens))
    got = W.prefill(c, tab, lens, starts, window, 4, q)
    parts = []
    for r, (n, at) in enumerate(zip(lens, np.cumsum([0] + lens))):
        pos, key = starts[r] + np.arange(n)[:, None], np.arange(total[r])[None]
        parts.append(squares(c, tab[r], (key <= pos) & ((key > pos - window) | (key < 4)), q[at:at + n], got[at:at + n]))
    held(parts)
    c.c.destroy()


@pytest.mark.parametrize("heads,batch,ctx,window", [(H128, 64, 900, 4096), (H128, 16, 3000, 4096), (H128, 4, 6000, 1024), (H64, 64, 900, 700)], ids=str)
def test_decode_rows(heads, batch, ctx, window):
    lens = [ctx + 17 * i for i in range(batch)]
    c = Step(heads, sum(n // 16 + 1 for n in lens), max_batch=batch, max_context=8192, seed=51)
    tab = c.tables([n + 1 for n in lens])
    q = c.queries(batch)
    got = W.decode(c, tab, lens, window, 4, q)
    held([squares(c, tab[r], (lambda key: (key > n - window) | (key < 4))(np.arange(n + 1)[None]), q[r:r + 1], got[r:r + 1]) for r, n in enumerate(lens)])
    c.c.destroy()


@pytest.mark.parametrize("heads,batch,ctx,draft", [(H128, 4, 900, 8), (H128, 32, 2300, 32), (H128, 8, 2000, 32), (H128, 64, 1000, 16), (H64, 32, 1000, 32)], ids=str)
def test_trees(heads, batch, ctx, draft):
    ctxs, lens = [ctx + 20 * i for i in range(batch)], [draft] * batch
    c = Step(heads, sum(-(-(n + draft) // 16) for n in ctxs), max_batch=batch, max_context=8192, seed=52)
    tab = c.tables([n + draft for n in ctxs])
    q = c.queries(batch * draft)
    got = T.tree(c, tab, ctxs, lens, None, q)
    parts = []
    for r, n in enumerate(ctxs):
        rows = slice(r * draft, (r + 1) * draft)
        parts.append(squares(c, tab[r], np.arange(n + draft)[None] <= n + np.arange(draft)[:, None], q[rows], got[rows]))
    held(parts)
    c.c.destroy()
