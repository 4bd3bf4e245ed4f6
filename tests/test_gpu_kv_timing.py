"""Launch timing of a chunk's attention: the copy and the attention are counted apart, so that the
kinds' times add up to the call's."""
import numpy as np
import pytest
import torch

from tests._step import DeviceCache, columns, device_rows, quantised, shape

pytestmark = pytest.mark.gpu


def test_kinds_add_up():
    import paper_2607_27600_gb300 as pkg
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(0)
    s, b, cap, counts = shape(8, 8, 128), 8, 8192, [65] * 8
    codes, exps = quantised(rng, 1, cap, 1, 128, 32)
    codes, exps = ({x: np.broadcast_to(y, (b, y.shape[1], 8) + y.shape[3:]) for x in "kv"} for y in (codes, exps))
    c, rows = DeviceCache(pkg, codes, exps, [8000] * 8, "slot"), device_rows(pkg, counts)
    dq, = columns([rng.standard_normal((sum(counts), 8, 128))], torch.bfloat16)
    out = torch.empty_like(dq)
    ws = cc.alloc_workspace(cc.cc_kv_attention_workspace_size(s, c.cache, rows))
    cc.cc_kv_attention(s, c.cache, 0, rows, dq, out, ws)
    a, z = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    cc.cc_timing_enable(True)
    try:
        torch.cuda._sleep(4_000_000)   # the host runs ahead
        a.record()
        cc.cc_kv_attention(s, c.cache, 0, rows, dq, out, ws)
        z.record()
        torch.cuda.synchronize()
        kinds = {k: x for k, x in cc.cc_timing_collect().items() if x[0]}
    finally:
        cc.cc_timing_enable(False)
    assert {k: x[0] for k, x in kinds.items()} == {"kv_dequant": 1, "kv_attention": 1}
    # (134 MB of codes: the copy is a good part of the call)
    assert kinds["kv_dequant"][1] > 0.1 * a.elapsed_time(z)
    assert sum(x[1] for x in kinds.values()) <= 1.02 * a.elapsed_time(z)
