"""The 4-bit cache without a GPU: its definition, and what the entry points refuse."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2601_11822_amd as rs
from tests import kv4_ref as R

P = 0x100000   # stands for a device pointer: refused calls touch nothing


def test_rounding_is_to_the_nearest_level_and_half_a_step_at_most():
    g = np.random.default_rng(1)
    x = R.f64(R.to_bf16_bits((g.standard_normal((400, 32)) * 2.0 ** g.integers(-60, 60, (400, 1))).astype(np.float32)))
    codes, scales = R.quantise(x)
    s = 2.0 ** (scales.astype(np.float64) - 127)
    amax = np.abs(x).max(-1, keepdims=True)
    assert (amax < 7 * s).all() and (amax >= 3.5 * s).all()
    y, r = R.values(codes, scales), np.abs(x) / s
    step = np.where(r < 2, 0.5, np.where(r < 4, 1.0, 2.0))
    assert (np.abs(x - y) <= 0.5 * step * s).all()
    assert np.array_equal(R.rounded(y), y)   # what the cache holds is held unchanged


def test_ties_signs_and_special_groups():
    x = np.zeros((4, 32))
    x[0, :9] = [6.99, 0.25, -0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -5.0]
    x[1, :2] = [7.0, 1.0]
    x[2, 3] = np.inf
    codes, scales = R.quantise(x)
    assert list(codes[0, 0, :9]) == [7, 0, 8, 2, 2, 4, 4, 6, 14] and list(scales[:, 0]) == [127, 128, 255, 2]
    assert list(R.values(codes, scales)[1, :2]) == [8.0, 1.0] and np.isnan(R.values(codes, scales)[2]).all()


def test_every_byte_of_a_block_has_one_place():
    for hd in (64, 128):
        seen = np.zeros(17 * hd, int)
        for t in range(16):
            for where in R.places(hd, t):
                seen[where] += 1
        assert (seen == 1).all() and rs.kv4_bytes(hd) == 17 * hd


def _ctx(kv4=True, **kw):
    base = dict(d_model=256, n_q_heads=4, n_kv_heads=2, head_dim=64, ffn_dim=688, n_layers=2, rms_eps=1e-5, rope_base=1e4, max_pos=1024,
                n_blocks=8, max_prefill_tokens=100, max_decode_batch=4, max_context=256, device=rs.RS_HOST_ONLY, kv4=kv4)
    base.update(kw)
    return rs.Context(**base)


def _refused(code, f, *a, **kw):
    with pytest.raises(rs.RapidServeError) as e:
        f(*a, **kw)
    assert e.value.code == code, str(e.value)


def test_contexts():
    _refused(rs.RS_ERR_BAD_ARG, _ctx, layer_stride=8 * 2 * 17 * 64 - 16)
    _refused(rs.RS_ERR_BAD_ARG, _ctx, layer_stride=8 * 2 * 17 * 64 + 8)
    _refused(rs.RS_ERR_BAD_ARG, _ctx, n_blocks=0)
    _refused(rs.RS_ERR_BAD_ARG, _ctx, head_dim=96)
    c = _ctx()
    assert list(c.kv_alloc(7, 33)) == [0, 1, 2] and c.kv_num_free() == 5
    c.destroy()
    lib = rs.load()
    assert lib.rs_init_kv4(None, None, None, None, ctypes.c_int32(-1), None) == rs.RS_ERR_BAD_ARG


ROWS = dict(side=0, layer=1, k=P, v=P, row_stride=128, block_tables=P, max_blk=4)
WRITE = dict(ROWS, cu_seqlens=[0, 5, 5, 30], start_pos=[3, 64, 39])
APPEND = dict(ROWS, ctx_lens=P, B=4)
DECODE = dict(layer=1, q=P, q_stride=256, out=P, out_stride=264, ctx_lens=P, block_tables=P, max_blk=4, B=4, max_ctx=64)
PREFILL = dict(layer=1, q=P, q_stride=256, out=P, out_stride=256, cu_seqlens=[0, 64], start_pos=None, block_tables=P, max_blk=4)


def _read(kw):
    kw = dict(kw)
    kw["k_out"], kw["v_out"] = kw.pop("k"), kw.pop("v")
    return kw


COMMON = [(dict(layer=2), -1), (dict(layer=-1), -1), (dict(block_tables=None), -1), (dict(max_blk=0), -4)]
SIDE = [(dict(side=2), -1), (dict(side=-1), -1)]
RUNS = [(dict(cu_seqlens=[1, 5]), -1), (dict(cu_seqlens=[0]), -1), (dict(cu_seqlens=list(range(66))), -1),
        (dict(cu_seqlens=[0, 5, 4]), -1), (dict(cu_seqlens=[0, 65]), -4)]
K = [(dict(k=None), -1), (dict(v=None), -1), (dict(k=P + 8), -1), (dict(v=P + 2), -1), (dict(row_stride=120), -1), (dict(row_stride=132), -1)]
STARTS = [(dict(cu_seqlens=[0, 5], start_pos=[60]), -4), (dict(cu_seqlens=[0, 5], start_pos=[-1]), -1),
          (dict(cu_seqlens=[0, 5], start_pos=[2**31 - 2]), -1), (dict(cu_seqlens=[0, 64], start_pos=[0]), -6),
          (dict(cu_seqlens=[0, 268435456], max_blk=1 << 25), -1), (dict(cu_seqlens=[0, 268434000], max_blk=1 << 25), -6)]
CALLS = (
    [("kv4_write", WRITE, ch, code) for ch, code in COMMON + SIDE + RUNS[:4] + K + STARTS + [({}, -6)]]
    + [("kv4_read", WRITE, ch, code) for ch, code in COMMON + SIDE + RUNS[:4] + K + STARTS + [({}, -6)]]
    + [("kv4_append", APPEND, ch, code) for ch, code in COMMON + SIDE + K + [(dict(ctx_lens=None), -1), (dict(B=0), -1), (dict(B=65536), -1), ({}, -6)]]
    + [("kv4_decode_attention", DECODE, ch, code) for ch, code in COMMON + [
        (dict(q=None), -1), (dict(out=None), -1), (dict(q=P + 8), -1), (dict(out=P + 4), -1), (dict(q_stride=248), -1), (dict(out_stride=260), -1),
        (dict(ctx_lens=None), -1), (dict(B=0), -1), (dict(B=5), -1), (dict(max_ctx=0), -1), (dict(max_ctx=257), -1), (dict(max_ctx=65), -4), ({}, -6)]]
    + [("kv4_prefill_attention", PREFILL, ch, code) for ch, code in COMMON + RUNS + [
        (dict(q=None), -1), (dict(out=None), -1), (dict(q_stride=250), -1), (dict(out_stride=0), -1), (dict(cu_seqlens=[0, 101], max_blk=100), -1),
        (dict(cu_seqlens=[0, 5], start_pos=[-16]), -1), (dict(cu_seqlens=[0, 5], start_pos=[60]), -4), ({}, -6)]])


@pytest.mark.parametrize("name,base,change,code", CALLS, ids=lambda v: str(v) if not isinstance(v, dict) or len(v) < 3 else "")
def test_refusals(name, base, change, code):
    """A code of -6 (RS_ERR_STATE): every argument is fine, and there is no device."""
    kw = dict(base)
    if name in ("kv4_write", "kv4_read") and "cu_seqlens" in change and "start_pos" not in change:
        kw["start_pos"] = None
    kw.update(change)
    c = _ctx()
    _refused(code, getattr(c, name), **(_read(kw) if name == "kv4_read" else kw))
    c.destroy()


def test_a_bf16_context_refuses_them_and_a_wrong_count_of_positions_is_seen():
    c = _ctx(kv4=False)
    for name, kw in (("kv4_write", WRITE), ("kv4_append", APPEND), ("kv4_read", _read(WRITE)), ("kv4_decode_attention", DECODE), ("kv4_prefill_attention", PREFILL)):
        _refused(rs.RS_ERR_STATE, getattr(c, name), **kw)
    c.destroy()
    c = _ctx()
    for cu in (np.array([0, 5, 5, 30]), torch.tensor([0, 5, 5, 30]), (0, 5, 5, 30)):
        _refused(rs.RS_ERR_STATE, c.kv4_write, **dict(WRITE, cu_seqlens=cu, start_pos=np.array([3, 64, 39], np.int32)))
    with pytest.raises(ValueError):
        c.kv4_write(**dict(WRITE, start_pos=[0]))
    c.destroy()
    lib = rs.load()
    assert lib.rs_kv4_write(None, 0, 0, None, None, ctypes.c_int64(0), None, None, 0, None, 0) == rs.RS_ERR_BAD_ARG
