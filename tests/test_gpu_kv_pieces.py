"""cc_kv_attention where the units of a chunk are cut into pieces for the SMs: a few long
units, more than SMs of nearly one length, very different ones, an empty memory and rows
without company.  Against the formula in 64 bits on the device; tolerances as
tests/test_gpu_kv_attention.py derives them."""
import numpy as np
import pytest
import torch

from tests._step import DeviceCache, columns, device_rows, quantised, shape, values

pytestmark = pytest.mark.gpu
TYPES = {"bf16": (torch.bfloat16, 2.0 ** -8, 2.0 ** -8), "f16": (torch.float16, 2.0 ** -11, 2.0 ** -11)}


def formula(q, k, v, lens, counts, memory):
    """Output, lse and sum_j p_j |V_j| of the rows (fp64, on the device)."""
    hq, group = q.shape[1], q.shape[1] // k.shape[2]
    out, lse, spread, at = torch.zeros_like(q), torch.full(q.shape[:2], -torch.inf).to(q), torch.zeros_like(q), 0
    for b, (n, m) in enumerate(zip(lens, counts)):
        end = n if memory else n + m
        for h in range(hq if end and m else 0):
            kk, vv = k[b, :end, h // group], v[b, :end, h // group]
            x = q[at:at + m, h] @ kk.T / q.shape[2] ** 0.5
            if not memory:
                row = torch.arange(m, device=q.device)[:, None]
                x = x.masked_fill(torch.arange(end, device=q.device)[None] > n + row, -torch.inf)
            p = torch.softmax(x, 1)
            out[at:at + m, h], spread[at:at + m, h] = p @ vv, p @ vv.abs()
            lse[at:at + m, h] = torch.logsumexp(x, 1)
        at += m
    return out, lse, spread


@pytest.mark.parametrize("memory", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,dh,layout,cap,lens,counts", [
    (8, 2, 64, "slot", 16384, [16000], [100]),
    (4, 1, 128, "paged", 8192, [8000], [131]),
    (32, 8, 64, "paged", 4352, [3000], [1280]),
    (14, 2, 64, "head", 5376, [5000, 0, 3, 900], [300, 1, 130, 64]),
    (8, 8, 64, "slot", 2048, [0, 1600, 1100, 128, 127], [129, 300, 260, 0, 1000]),
])
def test_pieces(hq, hkv, dh, layout, cap, lens, counts, dtype, memory):
    import paper_2607_27600_gb300 as pkg
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(cap + hq)
    s, b, n = shape(hq, hkv, dh), len(lens), sum(counts)
    codes, exps = {}, {}
    for x in "kv":
        codes[x], exps[x] = quantised(rng, b, cap, hkv, dh, 32)
    k, v = (torch.from_numpy(values(codes[x], exps[x])).cuda() for x in "kv")
    t, eps, p = TYPES[dtype]
    dq, = columns([rng.standard_normal((n, hq, dh)) * 1.5], t)
    c, rows = DeviceCache(pkg, codes, exps, lens, layout), device_rows(pkg, counts)
    ws = cc.alloc_workspace(cc.cc_kv_attention_workspace_size(s, c.cache, rows))
    got = []
    for fill in (0xFF, 0):   # the same bits, whatever the workspace held
        ws.fill_(fill)
        out, lse = torch.full((n, hq, dh), 7.0, dtype=t, device="cuda"), torch.full((n, hq), 7.0, device="cuda")
        cc.cc_kv_attention(s, c.cache, 0, rows, dq, out, ws, lse=lse, memory_only=memory)
        assert cc.cc_get_status() == cc.CC_OK
        got.append((out, lse))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    out, lse = (x.double() for x in got[0])
    want, want_lse, spread = formula(dq.double(), k, v, lens, counts, memory)
    assert ((out - want).abs() <= eps * want.abs() + 2 * p * spread + 1e-30).all()
    assert torch.equal(lse.isinf(), want_lse.isinf())
    f = want_lse.isfinite()
    assert ((lse - want_lse).abs()[f] <= 2.0 ** -12 + 2.0 ** -22 * want_lse[f].abs()).all()


def test_a_captured_chunk_is_planned_again_at_each_replay():
    import paper_2607_27600_gb300 as pkg
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(3)
    s, cap = shape(8, 2, 64), 6144
    codes, exps = {}, {}
    for x in "kv":
        codes[x], exps[x] = quantised(rng, 2, cap, 2, 64, 64)
    c, rows = DeviceCache(pkg, codes, exps, [0, 0], "slot"), device_rows(pkg, [300, 100])
    dq, = columns([rng.standard_normal((400, 8, 64))], torch.bfloat16)
    out = torch.empty(400, 8, 64, dtype=torch.bfloat16, device="cuda")
    ws = cc.alloc_workspace(cc.cc_kv_attention_workspace_size(s, c.cache, rows))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lens = ([0, 0], [5500, 9], [3, 6000], [4000, 4000])
    want = []
    for n in lens:
        with torch.cuda.stream(side):
            c.d["seq_len"].copy_(torch.tensor(n, dtype=torch.int32))
        cc.cc_kv_attention(s, c.cache, 0, rows, dq, out, ws, stream=side)
        with torch.cuda.stream(side):
            want.append(out.clone())
    cc.cc_graph_begin(side)
    cc.cc_kv_attention(s, c.cache, 0, rows, dq, out, ws, stream=side)
    graph = cc.cc_graph_end(side)
    for n, w in zip(lens, want):
        with torch.cuda.stream(side):
            c.d["seq_len"].copy_(torch.tensor(n, dtype=torch.int32))
            out.zero_()
        cc.cc_graph_launch(graph, side)
        with torch.cuda.stream(side):
            assert torch.equal(out, w)
    assert cc.cc_get_status(side) == cc.CC_OK
    cc.cc_graph_destroy(graph)
