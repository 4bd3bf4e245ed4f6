"""A row_start too short for the cache's batch is refused on the host (no GPU): the kernels read
batch + 1 entries of it."""
import types

import pytest

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("entries", [0, 1, 3])
def test_row_start_has_an_entry_more_than_sequences(entries):
    from paper_2607_27600_gb300 import cc
    cfg = cc.cc_model_cfg(1, 512, 8, 2, 64, 384, 1000, 1e4, 1e-5)
    cache = types.SimpleNamespace(c=cc.cc_kv_cache(batch=3))
    rows = types.SimpleNamespace(c=cc.cc_rows(4, 4, 1 << 20, None),
                                 row_start=torch.zeros(entries, dtype=torch.int32), pos=None)
    x = torch.zeros(4, 2, 64)
    for call in (lambda: cc.cc_kv_append(cfg, cache, 0, rows, x, x),
                 lambda: cc.cc_kv_attention_workspace_size(cfg, cache, rows),
                 lambda: cc.cc_kv_attention(cfg, cache, 0, rows, x, x, x),
                 lambda: cc.cc_kv_advance(cache, rows)):
        with pytest.raises(ValueError, match="row_start"):
            call()
