"""cc_kv_attention against the fp64 oracle (oracle/step.py): head groups and dims,
layouts, block sizes, row counts from one token to chunks, lengths at the edges of
tiles, blocks and pages, sequences without rows or slots, scales far apart, strides
and what lies past the ends; refusals and reports.

Tolerances.  The output is rounded to its type (unit roundoff: bf16 2^-8, fp16 2^-11).
Each probability is rounded once (fp16 2^-11; bf16, on the tile path, 2^-8) and its
score carries fp32 sums: that for the first and as much again for the second, of
A = sum_j p_j |V_j|.  lse: the scores' share, 2^-12, and fp32."""
import numpy as np
import pytest
import torch

import oracle
from tests._step import DeviceCache, columns, device_rows, quantised, shape, starts, values

pytestmark = pytest.mark.gpu
TYPES = {"bf16": (torch.bfloat16, 2.0 ** -8), "f16": (torch.float16, 2.0 ** -11)}


@pytest.fixture(scope="module")
def pkg():
    import paper_2607_27600_gb300 as p
    p.load_library()
    return p


def attend(pkg, s, c, counts, dq, memory=False, lse=True, pad=0):
    from paper_2607_27600_gb300 import cc
    n = len(dq)
    wide = torch.full((n, s.n_q_heads * s.head_dim + pad), 7.0, dtype=dq.dtype, device="cuda")
    out = wide[:, :s.n_q_heads * s.head_dim].view(n, s.n_q_heads, s.head_dim)
    ls = torch.full((n, s.n_q_heads), 7.0, device="cuda") if lse else None
    rows = device_rows(pkg, counts)
    ws = cc.alloc_workspace(cc.cc_kv_attention_workspace_size(s, c.cache, rows))
    ws.fill_(0xFF)   # NaN partials wherever nothing is written
    cc.cc_kv_attention(s, c.cache, 0, rows, dq, out, ws, lse=ls, memory_only=memory)
    assert (wide[:, s.n_q_heads * s.head_dim:] == 7).all()
    return out, ls


def check(got, ls, want, want_lse, spread, eps, tile=False):
    p = 2.0 ** (-8 if tile else -11)
    got = got.double().cpu().numpy()
    assert (np.abs(got - want) <= eps * np.abs(want) + 2 * p * spread + 1e-30).all(), \
        (np.abs(got - want) / (eps * np.abs(want) + 2 * p * spread + 1e-30)).max()
    if ls is not None:
        ls = ls.double().cpu().numpy()
        np.testing.assert_array_equal(np.isinf(ls), np.isinf(want_lse))
        f = np.isfinite(want_lse)
        assert (np.abs(ls - want_lse)[f] <= 2.0 ** -12 + 2.0 ** -22 * np.abs(want_lse[f])).all()


def junk(rng, codes, exps, ends, block):
    """NaN codes and any exponents past the ends."""
    for i, n in enumerate(ends):
        for x in "kv":
            codes[x][i, n:] = 0x7F | (rng.integers(0, 2, codes[x][i, n:].shape) << 7)
            exps[x][i, -(-n // block):] = rng.integers(0, 256, exps[x][i, -(-n // block):].shape)


EDGES = [0, 1, 14, 15, 16, 17, 62, 63, 64, 65, 126, 127, 128, 190, 254]
CASES = [
    # hq, hkv, dh, block, layout, dtype, cap, lens, counts
    (1, 1, 64, 16, "slot", "bf16", 256, EDGES, [1] * 15),
    (8, 2, 64, 128, "paged", "f16", 256, EDGES, [1] * 15),
    (7, 1, 128, 32, "head", "bf16", 256, EDGES, [1] * 15),
    (16, 2, 128, 64, "paged", "bf16", 256, EDGES, [1] * 15),            # 8 rows a unit
    (12, 1, 64, 16, "slot", "f16", 256, EDGES, [1] * 15),               # 12 rows
    (20, 1, 128, 64, "head", "bf16", 256, [0, 100, 255], [1, 1, 1]),    # 20 rows
    (72, 1, 64, 16, "paged", "bf16", 128, [0, 100], [1, 1]),            # three groups of rows
    (8, 2, 128, 16, "paged", "f16", 256, [0, 3, 250, 100, 77], [4, 0, 6, 3, 5]),
    (8, 2, 64, 32, "slot", "f16", 512, [0, 3, 250, 100, 400], [33, 0, 150, 3, 112]),
    (4, 1, 128, 128, "head", "f16", 2048, [1500], [300]),
    (8, 8, 64, 64, "paged", "bf16", 1024, [1000, 1, 0], [24, 16, 9]),
    (4, 4, 128, 64, "slot", "bf16", 2560, [2500, 2501, 9], [1, 1, 1]),  # several shares a unit
    (8, 1, 64, 16, "paged", "f16", 4096, [4000, 17], [1, 1]),
]


@pytest.mark.parametrize("memory", [False, True])
@pytest.mark.parametrize("hq,hkv,dh,block,layout,dtype,cap,lens,counts", CASES)
def test_matches_oracle(pkg, hq, hkv, dh, block, layout, dtype, cap, lens, counts, memory):
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(hq * 1000 + cap)
    s, b = shape(hq, hkv, dh), len(lens)
    codes, exps = {}, {}
    for n in "kv":
        codes[n], exps[n] = quantised(rng, b, cap, hkv, dh, block)
    ends = lens if memory else [n + m for n, m in zip(lens, counts)]
    junk(rng, codes, exps, ends, block)
    t, eps = TYPES[dtype]
    q = torch.from_numpy(rng.standard_normal((sum(counts), hq, dh)) * 1.5).to(t).double().numpy()
    dq, = columns([q], t, 24)
    c = DeviceCache(pkg, codes, exps, lens, layout)
    got, ls = attend(pkg, s, c, counts, dq, memory, pad=8)
    assert cc.cc_get_status() == cc.CC_OK
    want = oracle.attend_rows(q, values(codes["k"], exps["k"]), values(codes["v"], exps["v"]), lens,
                              starts(counts), memory)
    check(got, ls, *want, eps, tile=dtype == "bf16" and max(counts) > 32)
    again, _ = attend(pkg, s, c, counts, dq, memory, lse=False)
    assert torch.equal(again, got)   # the same bits, run to run


CHUNKS = [
    (8, 2, 64, 16, "paged", 512, [0, 130, 300], [200, 150, 64], 0),
    (4, 1, 128, 64, "head", 1024, [777], [130], 0),
    (7, 1, 128, 128, "slot", 384, [0, 1, 127, 128], [257, 64, 128, 129], 0),
    (16, 2, 64, 32, "paged", 256, [10, 0, 90, 256], [100, 40, 0, 0], 8),
    (3, 3, 128, 32, "paged", 2304, [2048], [72], 0),                    # key splits
]


@pytest.mark.parametrize("memory", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,dh,block,layout,cap,lens,counts,pad", CHUNKS)
def test_chunks_match_oracle(pkg, hq, hkv, dh, block, layout, cap, lens, counts, pad, dtype, memory):
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(hq * 1000 + cap)
    s, b = shape(hq, hkv, dh), len(lens)
    codes, exps = {}, {}
    for n in "kv":
        codes[n], exps[n] = quantised(rng, b, cap, hkv, dh, block)
    junk(rng, codes, exps, lens if memory else [n + m for n, m in zip(lens, counts)], block)
    t, eps = TYPES[dtype]
    q = torch.from_numpy(rng.standard_normal((sum(counts), hq, dh)) * 1.5).to(t).double().numpy()
    c = DeviceCache(pkg, codes, exps, lens, layout)
    got, ls = attend(pkg, s, c, counts, columns([q], t, 24)[0], memory, pad=pad)
    assert cc.cc_get_status() == cc.CC_OK
    want = oracle.attend_rows(q, values(codes["k"], exps["k"]), values(codes["v"], exps["v"]), lens,
                              starts(counts), memory)
    check(got, ls, *want, eps, tile=dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("counts", [[6, 2], [100, 40]])
def test_not_a_number_of_a_later_row(pkg, counts, dtype):
    """A NaN code among a new token's values reaches the rows that see it and no others."""
    rng = np.random.default_rng(12)
    s, cap, block, lens = shape(8, 2, 64), 256, 16, [120, 3]
    codes, exps = {}, {}
    for n in "kv":
        codes[n], exps[n] = quantised(rng, 2, cap, 2, 64, block)
    k, v = values(codes["k"], exps["k"]), values(codes["v"], exps["v"])
    t, eps = TYPES[dtype]
    q = torch.from_numpy(rng.standard_normal((sum(counts), 8, 64))).to(t).double().numpy()
    want = oracle.attend_rows(q, k, v, lens, starts(counts))
    row = counts[0] // 2
    codes["v"][0, lens[0] + row, 1, [7, 40]] = [0x7F, 0xFF]
    codes["v"][1, lens[1] + counts[1] - 1, 0, 63] = 0x7F
    c = DeviceCache(pkg, codes, exps, lens, "paged")
    got, ls = attend(pkg, s, c, counts, columns([q], t)[0])
    got = got.double()
    bad = torch.zeros(got.shape, dtype=torch.bool)
    bad[row:counts[0], 4:, [7, 40]] = True
    bad[-1, :4, 63] = True
    assert torch.equal(torch.isnan(got).cpu(), bad)
    got[bad] = torch.from_numpy(want[0])[bad].cuda()
    check(got, ls, *want, eps, tile=dtype == "bf16" and counts[0] > 32)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_scales_far_apart(pkg, dtype):
    """Value scales over 2^+-40 between blocks, key scales over 2^+-6, queries over
    the range of their type: the sums above and below keep their references apart."""
    rng = np.random.default_rng(3)
    s, cap, block = shape(4, 2, 64), 512, 16
    codes, exps = {}, {}
    for n in "kv":
        codes[n], exps[n] = quantised(rng, 2, cap, 2, 64, block)
    exps["v"] = (exps["v"].astype(int) + rng.integers(-40, 41, exps["v"].shape)).astype(np.uint8)
    exps["k"] = (exps["k"].astype(int) + rng.integers(-6, 3, exps["k"].shape)).astype(np.uint8)
    t, eps = TYPES[dtype]
    big = 2.0 ** rng.integers(-30, 2, (2, 4, 1)) if dtype == "bf16" else 2.0 ** rng.integers(-10, 2, (2, 4, 1))
    q = torch.from_numpy(rng.standard_normal((2, 4, 64)) * big).to(t).double().numpy()
    c = DeviceCache(pkg, codes, exps, [511, 300], "slot")
    got, ls = attend(pkg, s, c, [1, 1], columns([q], t)[0])
    want = oracle.attend_rows(q, values(codes["k"], exps["k"]), values(codes["v"], exps["v"]), [511, 300],
                              [0, 1, 2])
    if dtype == "f16":   # what fp16 cannot hold is no error
        inf = np.abs(want[0]) > 65504
        g = got.double().cpu().numpy()
        assert (np.abs(g[inf]) >= 65504).all()
        g[inf] = want[0][inf]
        got = torch.from_numpy(g)
        tiny = 2.0 ** -25 / eps
    else:
        tiny = 0.0
    check(got, ls, want[0], want[1], want[2] + tiny, eps)


def test_scales_at_the_ends_of_the_range(pkg):
    """Value scales of 2^-110 and 2^110 side by side, where the large ones have next to no
    weight and where they have all."""
    rng = np.random.default_rng(13)
    s, cap, block = shape(2, 1, 64), 256, 16
    codes, exps = {}, {}
    for n in "kv":
        codes[n], exps[n] = quantised(rng, 2, cap, 1, 64, block, (0.9, 1.1))
    big = np.arange(cap // block) % 3 == 1
    exps["v"][:, :, 0] = np.where(big, 237, 17)
    k = values(codes["k"], exps["k"]).copy()
    q = np.zeros((2, 2, 64))
    # sequence 0 shuns the blocks of large scale by 300 in score, sequence 1 seeks them
    codes["k"][:, :, 0, 0] = np.where(np.repeat(big, block), 0x7E, 0xFE)   # +-448
    exps["k"][:] = 127
    q[0, :, 0], q[1, :, 0] = -2.5, 2.5
    k, v = values(codes["k"], exps["k"]), values(codes["v"], exps["v"])
    c = DeviceCache(pkg, codes, exps, [255, 255], "slot")
    got, ls = attend(pkg, s, c, [1, 1], columns([q], torch.bfloat16)[0])
    want = oracle.attend_rows(q, k, v, [255, 255], [0, 1, 2])
    assert 2.0 ** -112 < np.abs(want[0][0]).max() < 2.0 ** -90 and np.abs(want[0][1]).max() > 2.0 ** 100
    check(got, ls, *want, 2.0 ** -8)


def test_one_key_dominates(pkg):
    """Scores over hundreds: the references rise late, early and not at all."""
    rng = np.random.default_rng(4)
    s, cap, block = shape(2, 1, 128), 1024, 32
    codes, exps = {}, {}
    for n in "kv":
        codes[n], exps[n] = quantised(rng, 3, cap, 1, 128, block, (0.9, 1.1))
    k = values(codes["k"], exps["k"])
    q = np.stack([np.stack([k[0, 1000, 0], -k[0, 5, 0]]), np.stack([k[1, 0, 0], k[1, 512, 0]]),
                  np.zeros((2, 128))]) * 40
    q = torch.from_numpy(q).to(torch.bfloat16).double().numpy()
    c = DeviceCache(pkg, codes, exps, [1023] * 3, "paged")
    got, ls = attend(pkg, s, c, [1, 1, 1], columns([q], torch.bfloat16)[0])
    want = oracle.attend_rows(q, k, values(codes["v"], exps["v"]), [1023] * 3, [0, 1, 2, 3])
    # scores of a few hundred: fp32 carries 2^-24 of their 128 terms' size, 2^13
    g = got.double().cpu().numpy()
    assert (np.abs(g - want[0]) <= 2.0 ** -8 * np.abs(want[0]) + 2.0 ** -9 * want[2]).all()
    assert (np.abs(ls.double().cpu().numpy() - want[1]) <= 2.0 ** -10 + 2.0 ** -20 * np.abs(want[1])).all()


def test_joins_with_attention_elsewhere(pkg):
    """The memory alone and the rows' own slots, joined by their lse, are the causal
    attention over both."""
    rng = np.random.default_rng(5)
    s, cap, block, lens, m = shape(4, 2, 64), 256, 16, [200, 0], 6
    codes, exps = {}, {}
    for n in "kv":
        codes[n], exps[n] = quantised(rng, 2, cap, 2, 64, block)
    q = torch.from_numpy(rng.standard_normal((2 * m, 4, 64))).half().double().numpy()
    c = DeviceCache(pkg, codes, exps, lens, "slot")
    dq, = columns([q], torch.float16)
    whole, wl = attend(pkg, s, c, [m, m], dq)
    part, pl = attend(pkg, s, c, [m, m], dq, memory=True)
    k, v = values(codes["k"], exps["k"]), values(codes["v"], exps["v"])
    own = [x[[0, 1]] for x in (k, v)]
    own = [np.stack([x[i, n:n + m] for i, n in enumerate(lens)]) for x in own]
    o2, l2, _ = oracle.attend_rows(q, own[0], own[1], [0, 0], [0, m, 2 * m])
    l1 = pl.double().cpu().numpy()
    w = 1 / (1 + np.exp(l1 - l2))[..., None]
    joined = part.double().cpu().numpy() * (1 - w) + o2 * w
    assert np.abs(joined - whole.double().cpu().numpy()).max() < 4e-3
    assert np.abs(np.logaddexp(l1, l2) - wl.double().cpu().numpy()).max() < 1e-3


def test_append_then_attend_step_by_step(pkg):
    """A prompt, then single tokens, each appended and attended: the attention of the
    values that the cache then holds."""
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(6)
    s, cap, block = shape(6, 2, 64), 128, 32
    codes, exps = {}, {}
    for n in "kv":
        codes[n], exps[n] = quantised(rng, 2, cap, 2, 64, block)
    lens = [0, 30]
    c = DeviceCache(pkg, codes, exps, lens, "paged")
    ws = None
    for counts in ([37, 5], [1, 1], [1, 1], [2, 0]):
        n = sum(counts)
        parts = [torch.from_numpy(rng.standard_normal((n, h, 64))).half().double().numpy() for h in (6, 2, 2)]
        dq, dk, dv = columns(parts, torch.float16)
        pos = np.concatenate([np.arange(m) + a for a, m in zip(lens, counts)])
        rows = device_rows(pkg, counts, pos)
        qr, out = torch.empty(n, 6, 64, dtype=torch.float16, device="cuda"), \
            torch.empty(n, 6, 64, dtype=torch.float16, device="cuda")
        cc.cc_kv_append(s, c.cache, 0, rows, dk, dv, dq, qr)
        ws = cc.alloc_workspace(cc.cc_kv_attention_workspace_size(s, c.cache, rows))
        cc.cc_kv_attention(s, c.cache, 0, rows, qr, out, ws)
        cc.cc_kv_advance(c.cache, rows)
        assert cc.cc_get_status() == cc.CC_OK
        k, v = values(c.get("k"), c.get("k_exp")), values(c.get("v"), c.get("v_exp"))
        want = oracle.attend_rows(qr.double().cpu().numpy(), k, v, lens, starts(counts))
        check(out, None, *want, 2.0 ** -11)
        lens = [a + m for a, m in zip(lens, counts)]
    assert c.d["seq_len"].cpu().tolist() == lens


def test_not_a_number(pkg):
    """A NaN code in a key that is seen makes the rows that see it 0, in a value NaN in its
    column; keys not seen do nothing."""
    rng = np.random.default_rng(7)
    s, cap, block = shape(2, 1, 64), 128, 16
    codes, exps = {}, {}
    for n in "kv":
        codes[n], exps[n] = quantised(rng, 1, cap, 1, 64, block)
    q = torch.from_numpy(rng.standard_normal((3, 2, 64))).half().double().numpy()
    dq, = columns([q], torch.float16)
    codes["k"][0, 62, 0, 9] = 0x7F          # the last row's own slot
    codes["v"][0, 10, 0, 5] = 0x7F
    c = DeviceCache(pkg, codes, exps, [60], "slot")
    got, ls = attend(pkg, s, c, [3], dq)
    got, ls = got.float().cpu().numpy(), ls.cpu().numpy()
    assert np.isnan(got[:2, :, 5]).all() and np.isfinite(np.delete(got[:2], 5, 2)).all()
    assert np.isfinite(ls[:2]).all()
    assert (got[2] == 0).all() and not np.isfinite(ls[2]).any()


def test_device_errors(pkg):
    """Bad rows, lengths and pages are reported; the other sequences are right."""
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(8)
    s, cap, block = shape(4, 2, 64), 256, 32
    codes, exps = {}, {}
    for n in "kv":
        codes[n], exps[n] = quantised(rng, 3, cap, 2, 64, block)
    k, v = values(codes["k"], exps["k"]), values(codes["v"], exps["v"])
    q = torch.from_numpy(rng.standard_normal((6, 4, 64))).half().double().numpy()
    dq, = columns([q], torch.float16)
    for lens, start, most, bad, table in (([10, 255, 20], [0, 2, 4, 6], 2, 1, None),
                                          ([10, 30, 20], [0, 2, 6, 4], 4, 2, None),
                                          ([10, 30, 20], [0, 1, 2, 6], 2, 2, None),
                                          ([10, 30, -7], [0, 2, 4, 6], 2, 2, None),
                                          ([10, 140, 20], [0, 2, 4, 6], 2, 1, 1)):
        c = DeviceCache(pkg, codes, exps, lens, "paged")
        if table is not None:
            c.d["block_table"][table, 1] = -3
        rows = pkg.Rows(6, torch.tensor(start, dtype=torch.int32, device="cuda"), None, most)
        out = torch.full((6, 4, 64), 7.0, dtype=torch.float16, device="cuda")
        ws = cc.alloc_workspace(cc.cc_kv_attention_workspace_size(s, c.cache, rows))
        cc.cc_kv_attention(s, c.cache, 0, rows, dq, out, ws)
        assert cc.cc_get_status() == cc.CC_ERR_DEVICE_ARG
        for i in range(3):
            if i == bad:
                continue
            sl = slice(start[i], start[i + 1])
            want = oracle.attend_rows(q[sl], k[i:i + 1], v[i:i + 1], [lens[i]], [0, start[i + 1] - start[i]])
            check(out[sl], None, *want, 2.0 ** -11)
        if table is not None:   # the slots of the bad page are not seen
            want = oracle.attend_rows(q[2:4], k[1:2], v[1:2], [128], [0, 2], True)
            check(out[2:4], None, *want, 2.0 ** -11)
