"""The profiler over a cache held in 4 bits."""
import numpy as np
import pytest
import torch

import rs_synth as S

pytestmark = pytest.mark.gpu


def test_a_table_measured_over_a_cache_in_4_bits():
    from paper_2601_11822_amd import profiler
    be, ce, dc = [4], [1024], [64, 128]
    rig = profiler.Rig(S.MID, be, ce, prefill_tokens=256, max_context=513, kv4=True)
    d = profiler.profile(rig, be, ce, dc, n_layers=2, steps=4, warmup=1)
    lat = np.array(d["lat_distinct_us"])
    assert lat.shape == (1, 1, 2) and (lat > 0).all() and (np.array(d["lat_over_us"]) > 0).all() and d["meta"]["kv_cache"] == "4-bit"
    assert "KV cache in 4 bits" in profiler.to_markdown(d)
    # the passes were over that cache: the calls on it are served, and what the prompt wrote can be read back
    W = S.MID.n_kv_heads * S.MID.head_dim
    k, v = (torch.zeros((256, W), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    torch.cuda.synchronize()
    rig.c.kv4_read(0, 0, k, v, W, [0, 256], None, rig.ptab, rig.max_blk)
    rig.c.sync(0)
    assert torch.isfinite(k).all() and k.abs().amax() > 0 and torch.isfinite(rig.yd).all()
    rig.c.destroy()
