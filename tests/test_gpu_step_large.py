"""The serving step over a pool whose offsets pass 32 bits, and captured into a graph."""
import numpy as np
import pytest
import torch

import oracle
from tests._step import columns, shape, starts, values

pytestmark = pytest.mark.gpu


def test_offsets_past_32_bits():
    """Pages at the two ends of pools of 5.4 GB each: appended and attended (one row, and a
    chunk on the tile kernel) as if they were small."""
    import paper_2607_27600_gb300 as pkg
    from paper_2607_27600_gb300 import cc
    s, page, block, n_pages, cap = shape(8, 8, 128), 128, 32, 41000, 384
    assert n_pages * page * s.n_kv_heads * s.head_dim > 2 ** 32
    table = np.array([[n_pages - 1, 0, n_pages - 2], [1, n_pages - 3, n_pages - 4]], np.int32)
    rng = np.random.default_rng(0)
    d = {n: [torch.empty(n_pages, page, 8, 128, dtype=torch.uint8, device="cuda")] for n in "kv"}
    d.update({n + "_exp": [torch.empty(n_pages, page // block, 8, dtype=torch.uint8, device="cuda")] for n in "kv"})
    d.update(kv_block=block, block_table=torch.from_numpy(table).cuda(), page_size=page,
             seq_len=torch.zeros(2, dtype=torch.int32, device="cuda"),
             tokens=torch.zeros(2, cap, dtype=torch.int32, device="cuda"),
             pos=torch.zeros(2, cap, dtype=torch.int32, device="cuda"))
    c = pkg.Cache(d)
    lens = [0, 0]
    for counts in ([300, 200], [1, 1]):
        n = sum(counts)
        parts = [torch.from_numpy(rng.standard_normal((n, 8, 128))).to(torch.bfloat16).double().numpy()
                 for _ in range(3)]
        q, k, v = columns(parts, torch.bfloat16)
        rows = pkg.Rows(n, torch.from_numpy(starts(counts)).cuda(), None, max(counts))
        qr, out = torch.empty(n, 8, 128, dtype=torch.bfloat16, device="cuda"), \
            torch.empty(n, 8, 128, dtype=torch.bfloat16, device="cuda")
        cc.cc_kv_append(s, c, 0, rows, k, v, q, qr)
        cc.cc_kv_attention(s, c, 0, rows, qr, out,
                           cc.alloc_workspace(cc.cc_kv_attention_workspace_size(s, c, rows)))
        cc.cc_kv_advance(c, rows)
        assert cc.cc_get_status() == cc.CC_OK
        pages = {x: d[x][0][torch.from_numpy(table).cuda().long()].cpu().numpy() for x in ("k", "v", "k_exp", "v_exp")}
        flat = {x: y.reshape(2, -1, *y.shape[3:]) for x, y in pages.items()}
        # (slots past the ends hold any bits)
        want, _, spread = oracle.attend_rows(qr.double().cpu().numpy(), values(flat["k"], flat["k_exp"]),
                                             values(flat["v"], flat["v_exp"]), lens, starts(counts))
        st = starts(counts)
        for i, m in enumerate(counts):   # V of the rows, to an e4m3 rounding
            got = values(flat["v"], flat["v_exp"])[i, lens[i]:lens[i] + m]
            x = parts[2][st[i]:st[i + 1]]
            assert (np.abs(got - x) <= np.abs(x) * 2.0 ** -4 + np.abs(x).max() * 2.0 ** -15).all()
        # bf16 output, and P in bf16 on the tiles (tests/test_gpu_kv_attention.py)
        off = np.abs(out.double().cpu().numpy() - want)
        assert (off <= 2.0 ** -8 * np.abs(want) + 2.0 ** -7 * spread).all()
        lens = [a + m for a, m in zip(lens, counts)]


def test_a_captured_step_replays_as_the_cache_grows():
    import paper_2607_27600_gb300 as pkg
    from paper_2607_27600_gb300 import cc
    s, cap, block = shape(4, 2, 64), 128, 16

    def fresh():
        return pkg.Cache({"k": [torch.zeros(2, cap, 2, 64, dtype=torch.uint8, device="cuda")],
                          "v": [torch.zeros(2, cap, 2, 64, dtype=torch.uint8, device="cuda")],
                          "k_exp": [torch.zeros(2, cap // block, 2, dtype=torch.uint8, device="cuda")],
                          "v_exp": [torch.zeros(2, cap // block, 2, dtype=torch.uint8, device="cuda")],
                          "kv_block": block, "seq_len": torch.tensor([0, 5], dtype=torch.int32, device="cuda"),
                          "tokens": torch.zeros(2, cap, dtype=torch.int32, device="cuda"),
                          "pos": torch.arange(cap, dtype=torch.int32, device="cuda").repeat(2, 1).contiguous()})

    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(40, 2, 8, 64, generator=g, device="cuda").to(torch.bfloat16)
    now = torch.empty(2, 8, 64, dtype=torch.bfloat16, device="cuda")
    rows = pkg.Rows(2)
    q, out = torch.empty(2, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    ids, lp = torch.empty(2, 3, dtype=torch.int32, device="cuda"), torch.empty(2, 3, device="cuda")

    def step(cache, ws, stream):
        cc.cc_kv_append(s, cache, 0, rows, now[:, 4:6], now[:, 6:], now[:, :4], q, stream=stream)
        cc.cc_kv_attention(s, cache, 0, rows, q, out, ws, stream=stream)
        cc.cc_kv_advance(cache, rows, stream=stream)
        cc.cc_token_logprobs(out.view(2, 256), top_ids=ids, top_logprob=lp, stream=stream)

    got = []
    for captured in (False, True):
        cache = fresh()
        ws = cc.alloc_workspace(cc.cc_kv_attention_workspace_size(s, cache, rows))
        side, graph = torch.cuda.Stream(), None
        side.wait_stream(torch.cuda.current_stream())
        if captured:
            cc.cc_graph_begin(side)
            step(cache, ws, side)
            graph = cc.cc_graph_end(side)
        seen = []
        for i in range(40):
            with torch.cuda.stream(side):
                now.copy_(x[i])
            if captured:
                cc.cc_graph_launch(graph, side)
            else:
                step(cache, ws, side)
            with torch.cuda.stream(side):
                seen.append((out.clone(), ids.clone(), lp.clone()))
        assert cc.cc_get_status(side) == cc.CC_OK
        assert cache.d["seq_len"].tolist() == [40, 45]
        got.append(seen)
        if captured:
            cc.cc_graph_destroy(graph)
    for a, b in zip(*got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
