"""The manager's table for a cache held in 4 bits: measured over one, and refused over the other kind (no GPU)."""
import json

import pytest

from paper_2601_11822_amd import profiler, serve_bench

TABLE = {"batch_edges": [16], "ctx_edges": [1024], "decode_cus": [64], "lat_distinct_us": [[[10]]], "lat_over_us": [[20]]}


class Stop(Exception):
    pass


def serve(monkeypatch, seen, *argv):
    """serve_bench up to the point where it makes the model."""
    class Rig:
        def __init__(self, *a, kv4=False, **kw):
            seen["rig"] = kv4
            self.kv_cache = "4-bit" if kv4 else "bf16"
            self.c = self

        def destroy(self):
            pass

    def model(*a, kv4=False, **kw):
        seen["model"] = kv4
        raise Stop

    monkeypatch.setattr(profiler, "Rig", Rig)
    monkeypatch.setattr(profiler, "profile", lambda rig, *a, **kw: dict(TABLE, meta={"kv_cache": rig.kv_cache}))
    monkeypatch.setattr(serve_bench, "build_model", model)
    serve_bench.main(["--policy", "manager", "--requests", "2", "--layers", "2", *argv])


@pytest.mark.parametrize("kv4", [False, True])
def test_the_measured_table_is_of_the_served_cache(monkeypatch, kv4):
    seen = {}
    with pytest.raises(Stop):
        serve(monkeypatch, seen, "--profile", "measure", *(["--kv4"] if kv4 else []))
    assert seen == {"rig": kv4, "model": kv4}


@pytest.mark.parametrize("meta,kv4,fine", [(None, False, True), (None, True, False), ("bf16", False, True), ("bf16", True, False),
                                           ("4-bit", True, True), ("4-bit", False, False)])
def test_a_table_of_the_other_cache_is_refused(monkeypatch, tmp_path, capsys, meta, kv4, fine):
    path = tmp_path / "table.json"
    path.write_text(json.dumps(TABLE if meta is None else dict(TABLE, meta={"kv_cache": meta})))
    with pytest.raises(Stop if fine else SystemExit):
        serve(monkeypatch, {}, "--profile", str(path), *(["--kv4"] if kv4 else []))
    assert fine or "KV cache" in capsys.readouterr().err
    assert profiler.load_profile(str(path), 1000) is not None   # who does not ask is not refused
