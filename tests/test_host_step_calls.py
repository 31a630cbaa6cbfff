"""What the calls on parts of a step refuse, without a GPU."""
import pytest

import paper_2601_11822_amd as rs

P = 0x100000   # stands for a device pointer: refused calls touch nothing


def _ctx(**kw):
    base = dict(d_model=256, n_q_heads=4, n_kv_heads=2, head_dim=64, ffn_dim=688, n_layers=2, rms_eps=1e-5, rope_base=1e4, max_pos=1024,
                n_blocks=8, max_prefill_tokens=100, max_decode_batch=4, max_context=256, device=rs.RS_HOST_ONLY, k_pool=P, v_pool=P)
    base.update(kw)
    return rs.Context(**base)


CALLS = {
    "window_decode_attention": dict(layer=0, q=P, q_stride=256, out=P, out_stride=256, ctx_lens=P, block_tables=P, max_blk=16, B=4, max_ctx=256, window=64, sinks=4),
    "window_prefill_attention": dict(layer=0, q=P, q_stride=256, out=P, out_stride=256, cu_seqlens=[0, 40, 60], start_pos=[0, 5], block_tables=P, max_blk=16,
                                     window=64, sinks=4),
    "tree_attention": dict(layer=0, q=P, q_stride=256, out=P, out_stride=256, ctx_lens=P, cu_rows=P, masks=P, block_tables=P, max_blk=16, B=4, max_rows=64,
                           max_draft=64, max_ctx=256),
    "kv_plan": dict(side=1, lens=P, n_new=P, n_held=P, block_tables=P, max_blk=16, B=4, free_ids=P, free_cap=8, n_free=P, max_rows=64, cu_rows=P, positions=P,
                    slots=P, n_held_out=P, n_free_out=P, parents=P, parent_stride=64, masks=P),
    "kv_store": dict(side=1, layer=0, qkv=P, row_stride=512, q_out=P, q_stride=256, positions=P, slots=P, max_rows=64, n_rows=P, n_axes=2, pair_axis=[0, 1] * 16),
    "kv_compact": dict(side=1, layer=0, n_layers=2, ctx_lens=P, keep=P, keep_stride=64, keep_lens=P, block_tables=P, max_blk=16, B=4),
}
A, K, S = rs.RS_ERR_BAD_ARG, rs.RS_ERR_BAD_BLOCK, rs.RS_ERR_STATE
ROWS = [(A, dict(q=0)), (A, dict(q=P + 8)), (A, dict(q_stride=255)), (A, dict(q_stride=260)), (A, dict(q_stride=248)), (A, dict(out=0)), (A, dict(out=P + 2)),
        (A, dict(out_stride=255)), (A, dict(layer=2)), (A, dict(layer=-1)), (A, dict(block_tables=0)), (A, dict(block_tables=P + 2)), (K, dict(max_blk=0)),
        (K, dict(max_blk=1 << 27))]
BATCH = [(A, dict(ctx_lens=0)), (A, dict(ctx_lens=P + 1)), (A, dict(B=0)), (A, dict(B=5)), (A, dict(max_ctx=0)), (A, dict(max_ctx=257)), (K, dict(max_blk=15))]
WINDOW = [(A, dict(window=0)), (A, dict(window=-1)), (A, dict(sinks=-1))]
REFUSED = {
    "window_decode_attention": ROWS + BATCH + WINDOW,
    "window_prefill_attention": ROWS + WINDOW + [(A, dict(cu_seqlens=[1, 2, 3])), (A, dict(cu_seqlens=[0, 5, 4])), (A, dict(cu_seqlens=[0], start_pos=None)),
                                                 (A, dict(cu_seqlens=[0] * 66, start_pos=None)), (A, dict(start_pos=[0, -1])), (A, dict(cu_seqlens=[0, 40, 101])),
                                                 (K, dict(start_pos=[217, 0])), (A, dict(start_pos=[2 ** 31 - 50, 0]))],
    "tree_attention": ROWS + BATCH + [(A, dict(cu_rows=0)), (A, dict(cu_rows=P + 2)), (A, dict(masks=P + 4)), (A, dict(max_draft=0)), (A, dict(max_draft=65)),
                                      (A, dict(max_rows=-1))],
    "kv_plan": [(A, {n: v}) for n in ("lens", "n_new", "n_held", "block_tables", "free_ids", "n_free", "cu_rows", "positions", "slots", "n_held_out", "n_free_out")
                for v in (0, P + 2)] + [(A, dict(side=2)), (A, dict(side=-1)), (K, dict(max_blk=0)), (K, dict(max_blk=1 << 27)), (A, dict(B=0)), (A, dict(B=65536)),
                                        (A, dict(free_cap=-1)), (A, dict(max_rows=-1)), (A, dict(parents=P + 1)), (A, dict(parent_stride=0)),
                                        (A, dict(parent_stride=65)), (A, dict(masks=P + 4)), (A, dict(parents=None))],
    "kv_store": [(A, dict(side=2)), (A, dict(layer=2)), (A, dict(qkv=0)), (A, dict(qkv=P + 8)), (A, dict(row_stride=504)), (A, dict(row_stride=516)),
                 (A, dict(q_out=P + 8)), (A, dict(q_stride=248)), (A, dict(positions=0)), (A, dict(positions=P + 2)), (A, dict(slots=0)), (A, dict(n_rows=P + 2)),
                 (A, dict(n_axes=0)), (A, dict(n_axes=5)), (A, dict(n_axes=1)), (A, dict(pair_axis=None)), (A, dict(pair_axis=[0, 2] * 16)), (A, dict(max_rows=0))],
    "kv_compact": [(A, dict(side=2)), (A, dict(layer=1)), (A, dict(layer=-1)), (A, dict(n_layers=0)), (A, dict(n_layers=3)), (A, dict(ctx_lens=0)), (A, dict(keep=0)),
                   (A, dict(keep=P + 2)), (A, dict(keep_lens=0)), (A, dict(keep_stride=0)), (A, dict(keep_stride=65)), (A, dict(block_tables=0)), (K, dict(max_blk=0)),
                   (A, dict(B=0)), (A, dict(B=65536))],
}


def _code(c, name, **kw):
    with pytest.raises(rs.RapidServeError) as e:
        getattr(c, name)(**{**CALLS[name], **kw})
    return e.value.code


@pytest.mark.parametrize("name", CALLS)
def test_refusals(name):
    c = _ctx()
    assert _code(c, name) == S   # a host-only context: the last check, behind all of the arguments
    for code, kw in REFUSED[name]:
        assert _code(c, name, **kw) == code, kw
    c.destroy()
    lib = rs.load()
    assert getattr(lib, "rs_" + name)(*[0] * len(rs._STEP_ARGS["rs_" + name])) == A   # no context


@pytest.mark.parametrize("name", CALLS)
def test_a_cache_held_in_4_bits(name):
    c = _ctx(k_pool=None, v_pool=None, kv4=True)
    if name == "kv_plan":   # touches no cache: refused for the missing GPU alone
        assert _code(c, name) == S and _code(c, name, B=0) == A
    else:
        assert _code(c, name, layer=7) == S
    c.destroy()


@pytest.mark.parametrize("name", [n for n in CALLS if n != "kv_plan"])
def test_pools_that_are_not_aligned(name):
    for kw in (dict(k_pool=P + 2), dict(v_pool=P + 8), dict(layer_stride=8 * 16 * 2 * 64 + 4)):
        c = _ctx(**kw)
        assert _code(c, name) == A
        c.destroy()


def test_more_rows_than_a_launch_has_threads_for():
    c = _ctx(n_q_heads=16 * 2048, n_kv_heads=2048, max_decode_batch=65535, n_layers=1)
    W = 16 * 2048 * 64
    assert _code(c, "tree_attention", q_stride=W, out_stride=W, B=65535) == A
    assert _code(c, "kv_store", row_stride=W + 2 * 2048 * 64, q_stride=W, max_rows=2 ** 31 - 1) == A
    assert _code(c, "kv_compact", n_layers=1, B=65535) == A and _code(c, "kv_compact", n_layers=1, B=8000) == S
    c.destroy()


def test_axes_of_another_length():
    c = _ctx()
    with pytest.raises(ValueError):
        c.kv_store(**{**CALLS["kv_store"], "pair_axis": [0, 1] * 32})
    c.destroy()
