"""cc_kv_append and cc_kv_advance against the fp64 oracle (oracle/step.py): every
format and layout, block sizes, input types, chunks at the edges of blocks and
pages, empty sequences, rescaled blocks, zeros, infinities and NaN, what is
refused and what is reported.

Tolerances.  A rotated value carries fp32 rounding of the angle (a turn to 2^-25:
2e-7), of cos and sin and of two products: below 2^-20 of its pair's radius.  A
code is the nearest to the exact quotient, or one that is farther by no more than
that.  Exponents are equal: their bound is computed without an angle."""
import numpy as np
import pytest
import torch

import oracle
from tests._step import DeviceCache, LAYOUTS, columns, device_rows, quantised, shape, starts, values

pytestmark = pytest.mark.gpu
ANGLE = 2.0 ** -20
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module")
def pkg():
    import paper_2607_27600_gb300 as p
    p.load_library()
    return p


def inputs(rng, s, counts, dtype, wild=False):
    """q, k, v as float64 of values that dtype holds, and their device columns."""
    n = int(sum(counts))
    parts = []
    for heads in (s.n_q_heads, s.n_kv_heads, s.n_kv_heads):
        x = rng.standard_normal((n, heads, s.head_dim))
        if wild:   # magnitudes of each row and head over 2^24
            x *= 2.0 ** rng.integers(-12, 12, (n, heads, 1))
        parts.append(torch.from_numpy(x).to(dtype).double().numpy())
    return parts, columns(parts, dtype, 8)


def check_codes(got, want, exact, exps, radius, written):
    """Codes at `written` slots: as near to the exact value as the nearest, but for the
    rotation's rounding; elsewhere untouched."""
    np.testing.assert_array_equal(got[~written], want[~written])
    block = got.shape[1] // exps.shape[1]
    scale = (2.0 ** (np.repeat(exps.astype(int), block, 1) - 127.0))[..., None]
    g, w = oracle.e4m3_decode(got) * scale, oracle.e4m3_decode(want) * scale
    new = written & ~np.isnan(exact).all((2, 3))
    off = np.abs(g[new] - exact[new]) - np.abs(w[new] - exact[new])
    assert (np.isnan(g[new]) == np.isnan(w[new])).all()
    assert (np.nan_to_num(off) <= 2 * ANGLE * radius[new] + 1e-300).all(), np.nanmax(off)


CASES = [
    # hq, hkv, dh, block, layout, dtype, lens, counts
    (4, 2, 64, 16, "slot", "bf16", [0, 1, 15, 16, 17, 100], [1, 1, 1, 1, 1, 1]),
    (7, 1, 128, 32, "paged", "bf16", [0, 31, 33, 127, 128, 200], [40, 1, 95, 2, 128, 0]),
    (8, 4, 64, 64, "head", "f16", [5, 0, 64, 190], [130, 3, 64, 2]),
    (2, 2, 128, 128, "paged", "f32", [0, 127, 129, 250], [256, 1, 100, 5]),
    (6, 3, 64, 128, "slot", "f32", [3, 77], [250, 0]),
    (5, 1, 128, 16, "head", "bf16", [9, 0, 256], [17, 256, 0]),
]


@pytest.mark.parametrize("hq,hkv,dh,block,layout,dtype,lens,counts", CASES)
@pytest.mark.parametrize("wild", [False, True])
def test_block_append_matches_oracle(pkg, hq, hkv, dh, block, layout, dtype, lens, counts, wild):
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(hq * 100 + block)
    s, b, cap = shape(hq, hkv, dh), len(lens), 256
    codes, exps = {}, {}
    for n in "kv":
        codes[n], exps[n] = quantised(rng, b, cap, hkv, dh, block)
    # what lies past the ends holds any bits, its exponents too
    for i, n in enumerate(lens):
        for x in "kv":
            codes[x][i, n:] = rng.integers(0, 256, codes[x][i, n:].shape)
            exps[x][i, -(-n // block):] = rng.integers(0, 256, exps[x][i, -(-n // block):].shape)
    (q, k, v), (dq, dk, dv) = inputs(rng, s, counts, TYPES[dtype], wild)
    pos = rng.integers(0, 131072, len(q))
    c = DeviceCache(pkg, codes, exps, lens, layout)
    q_out = torch.full((len(q), hq, dh), 7.0, dtype=TYPES[dtype], device="cuda")
    cc.cc_kv_append(s, c.cache, 0, device_rows(pkg, counts, pos), dk, dv, dq, q_out)
    assert cc.cc_get_status() == cc.CC_OK
    st = starts(counts)
    kr, qr = oracle.rotate_rows(s, k, pos), oracle.rotate_rows(s, q, pos)
    written = np.zeros((b, cap), bool)
    for i, (n, m) in enumerate(zip(lens, counts)):
        written[i, n // block * block if m else n:n + m] = True
    radius = np.zeros((b, cap, hkv, dh))
    for i, (n, m) in enumerate(zip(lens, counts)):
        r = np.hypot(k[st[i]:st[i + 1], :, :dh // 2], k[st[i]:st[i + 1], :, dh // 2:])
        radius[i, n:n + m] = np.concatenate([r, r], -1)
    for name, x, bound, rad in (("k", kr, oracle.k_bound(k), radius), ("v", v, oracle.v_bound(v), 0 * radius)):
        wc, we, exact = oracle.append_blocks(codes[name], exps[name], block, lens, st, x, bound)
        np.testing.assert_array_equal(c.get(name + "_exp"), we)
        got = c.get(name)
        check_codes(got, wc, exact, we, rad, written)
        old = written & np.isnan(exact).all((2, 3))   # rescaled, or as they were
        np.testing.assert_array_equal(got[old], wc[old])
    r = np.hypot(q[..., :dh // 2], q[..., dh // 2:])
    eps = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 0.0}[dtype]   # unit roundoffs
    # (fp16: subnormals round to multiples of 2^-24)
    tol = np.abs(qr) * eps + (ANGLE + eps * ANGLE) * np.concatenate([r, r], -1) + (2.0 ** -25 if dtype == "f16" else 0)
    got = q_out.double().cpu().numpy()
    fits = np.abs(qr) < 65504 if dtype == "f16" else np.ones(qr.shape, bool)
    assert (np.abs(got - qr) <= tol)[fits].all()
    assert c.d["seq_len"].cpu().tolist() == list(lens)   # until cc_kv_advance


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_other_formats(pkg, layout, fmt):
    """A bf16 cache holds the rounded rows; one scale a layer, codes of value / scale."""
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(5)
    s, lens, counts, cap = shape(4, 2, 64), [0, 33, 100], [70, 0, 28], 128
    q, k, v = inputs(rng, s, counts, torch.bfloat16)[0]
    dq, dk, dv = columns([q, k, v], torch.bfloat16)
    if fmt == "bf16":
        raw = {n: torch.randn(3, cap, 2, 64).to(torch.bfloat16) for n in "kv"}
        c = DeviceCache(pkg, raw, None, lens, layout)
    else:
        raw = {n: rng.integers(0, 127, (3, cap, 2, 64)).astype(np.uint8) for n in "kv"}
        c = DeviceCache(pkg, raw, None, lens, layout, scale=[(0.03, 0.07)])
    before = {n: c.get(n) for n in "kv"}
    pos = rng.integers(0, 9000, len(q))
    cc.cc_kv_append(s, c.cache, 0, device_rows(pkg, counts, pos), dk, dv)
    assert cc.cc_get_status() == cc.CC_OK
    st, kr = starts(counts), oracle.rotate_rows(s, k, pos)
    for n, x, sc in (("k", kr, 0.03), ("v", v, 0.07)):
        got = c.get(n)
        for i, (a, m) in enumerate(zip(lens, counts)):
            new, old = got[i, a:a + m], np.delete(got[i], np.arange(a, a + m), 0)
            np.testing.assert_array_equal(old, np.delete(before[n][i], np.arange(a, a + m), 0))
            want = x[st[i]:st[i + 1]]
            r = np.hypot(want[..., :32], want[..., 32:])
            r = np.concatenate([r, r], -1)
            if fmt == "bf16":
                assert (np.abs(new - want) <= 2.0 ** -8 * np.abs(want) + 1.01 * ANGLE * r).all()
            else:   # (value * (1 / scale): two more fp32 roundings)
                near = oracle.kv_quantize(want, np.float32(sc))
                off = np.abs(oracle.e4m3_decode(new.astype(np.uint8)) * np.float32(sc) - want) - np.abs(near - want)
                assert (off <= 2 * (ANGLE + 2.0 ** -22) * r).all()


def test_positions_follow_and_advance(pkg):
    """Without positions a row follows the cache's last one; cc_kv_advance records them
    and the tokens, and the next step's rows follow those."""
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(6)
    s, lens, cap, block = shape(4, 2, 64), [0, 20, 5], 64, 16
    zero = {n: np.zeros((3, cap, 2, 64), np.uint8) for n in "kv"}
    ones = {n: np.full((3, cap // block, 2), 118, np.uint8) for n in "kv"}
    pos0 = np.zeros((3, cap), np.int32)
    pos0[1, :20], pos0[2, :5] = np.arange(20) * 3 + 7, [0, 5, 6, 7, 90]
    c = DeviceCache(pkg, zero, ones, lens, "slot", pos=pos0)
    have = [0, 65, 91]
    for counts in ([3, 0, 2], [1, 1, 1]):
        q, k, v = inputs(rng, s, counts, torch.float32)[0]
        dq, dk, dv = columns([q, k, v], torch.float32)
        pos = np.concatenate([np.arange(m) + h for m, h in zip(counts, have)])
        rows = device_rows(pkg, counts) if counts[1] == 0 else pkg.Rows(3)   # (one each: no row_start)
        q_out = torch.empty_like(dq).contiguous()
        cc.cc_kv_append(s, c.cache, 0, rows, dk, dv, dq, q_out)
        tok = torch.arange(100, 100 + len(q), dtype=torch.int32, device="cuda")
        cc.cc_kv_advance(c.cache, rows, tok)
        assert cc.cc_get_status() == cc.CC_OK
        qr = oracle.rotate_rows(s, q, pos)
        r = np.hypot(q[..., :32], q[..., 32:])
        assert (np.abs(q_out.double().cpu().numpy() - qr) <= ANGLE * np.concatenate([r, r], -1)).all()
        p, t, at = c.d["pos"].cpu().numpy(), c.d["tokens"].cpu().numpy(), 0
        for i, m in enumerate(counts):
            assert p[i, lens[i]:lens[i] + m].tolist() == list(range(have[i], have[i] + m))
            assert t[i, lens[i]:lens[i] + m].tolist() == list(range(100 + at, 100 + at + m))
            at += m
        lens = [n + m for n, m in zip(lens, counts)]
        have = [h + m for h, m in zip(have, counts)]
        assert c.d["seq_len"].cpu().tolist() == lens


def test_no_rotation_in_place_and_scaled_frequencies(pkg):
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(7)
    s = shape(4, 2, 64, 5e5, (8.0, 1.0, 4.0, 8192))
    codes, exps = quantised(rng, 1, 64, 2, 64, 32)
    both = {"k": codes, "v": codes.copy()}, {"k": exps, "v": exps.copy()}
    counts, pos = [40], np.arange(40) + 5000
    for rotate in (False, True):
        c = DeviceCache(pkg, *both, [10], "slot")
        (q, k, v), (dq, dk, dv) = inputs(rng, s, counts, torch.bfloat16)
        cc.cc_kv_append(s, c.cache, 0, device_rows(pkg, counts, pos), dk, dv, dq, dq, rotate=rotate)
        assert cc.cc_get_status() == cc.CC_OK
        want = oracle.rotate_rows(s, q, pos) if rotate else q
        r = np.hypot(q[..., :32], q[..., 32:])
        tol = 2.0 ** -8 * np.abs(want) + 1.01 * ANGLE * np.concatenate([r, r], -1) if rotate else 0
        assert (np.abs(dq.double().cpu().numpy() - want) <= tol).all()
        if not rotate:
            wc, we, _ = oracle.append_blocks(codes, exps, 32, [10], starts(counts), k, oracle.k_bound(k))
            np.testing.assert_array_equal(c.get("k"), wc)
            np.testing.assert_array_equal(c.get("k_exp"), we)


def test_zeros_infinities_and_nan(pkg):
    """Zeros leave an older exponent alone; infinities and NaN become the NaN code and
    take no part in it; the largest and smallest fp32 magnitudes keep in range."""
    from paper_2607_27600_gb300 import cc
    s, cap, block = shape(2, 1, 64), 64, 16
    zero = {n: np.zeros((1, cap, 1, 64), np.uint8) for n in "kv"}
    some = {n: np.full((1, 4, 1), 90, np.uint8) for n in "kv"}
    c = DeviceCache(pkg, zero, some, [3], "slot")
    x = np.zeros((40, 1, 64), np.float32)
    x[13:29] = np.random.default_rng(8).standard_normal((16, 1, 64))   # slots 16 .. 31
    x[14, 0, 3], x[15, 0, 40], x[16, 0, 5] = np.inf, -np.inf, np.nan
    x[29, 0, :2] = [3.0e38, -1e-38]                                    # slots 32 .. 42
    t = torch.from_numpy(x).cuda()
    cc.cc_kv_append(s, c.cache, 0, device_rows(pkg, [40], np.arange(40)), t, t, rotate=False)
    assert cc.cc_get_status() == cc.CC_OK
    x64 = x.astype(np.float64)
    for n, bound in (("k", oracle.k_bound(x64)), ("v", oracle.v_bound(x64))):
        wc, we, _ = oracle.append_blocks(zero[n], some[n], block, [3], [0, 40], x64, bound)
        np.testing.assert_array_equal(c.get(n + "_exp"), we)
        assert we[0, 0, 0] == 90 and we[0, 2, 0] >= 246
        np.testing.assert_array_equal(c.get(n) & 0x7F, wc & 0x7F)   # (a NaN's sign may differ)
        assert (oracle.e4m3_decode(c.get(n)[0, 17:20]) != oracle.e4m3_decode(c.get(n)[0, 17:20])).sum() == 3


def test_device_errors(pkg):
    """A sequence past cap, with rows out of order or too many, a bad length, a bad
    page and a negative position are reported; the other sequences are written."""
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(9)
    s, cap, block = shape(4, 2, 64), 128, 32

    def run(lens, start, max_rows, bad, pos=None, table=None):
        codes, exps = quantised(rng, 3, cap, 2, 64, block)
        c = DeviceCache(pkg, {"k": codes, "v": codes.copy()}, {"k": exps, "v": exps.copy()}, lens,
                        "paged" if table is not None else "slot")
        if table is not None:
            c.d["block_table"][table, 0] = 99
        x = torch.randn(6, 2, 64, device="cuda")
        p = torch.arange(6, dtype=torch.int32, device="cuda") if pos is None else pos
        rows = pkg.Rows(6, torch.tensor(start, dtype=torch.int32, device="cuda"), p, max_rows)
        cc.cc_kv_append(s, c.cache, 0, rows, x, x)
        assert cc.cc_get_status() == cc.CC_ERR_DEVICE_ARG
        assert cc.cc_get_status() == cc.CC_OK
        got = c.get("v")
        for i in range(3):
            same = (got[i] == codes[i]).all()
            assert same == (i in bad), (i, bad)
        if table is None and pos is None:
            cc.cc_kv_advance(c.cache, rows)
            assert cc.cc_get_status() == cc.CC_ERR_DEVICE_ARG
            want = [n if i in bad else n + start[i + 1] - start[i] for i, n in enumerate(lens)]
            assert c.d["seq_len"].cpu().tolist() == want

    run([10, 127, 20], [0, 2, 4, 6], 2, {1})            # past cap
    run([10, 30, 20], [0, 4, 2, 6], 4, {1})             # out of order
    run([10, 30, 20], [0, 1, 2, 6], 2, {2})             # more than max_rows
    run([10, 30, 20], [0, 2, 4, 9], 6, {2})             # past n_rows
    run([-1, 30, 20], [0, 2, 4, 6], 2, {0})
    run([10, 129, 20], [0, 2, 4, 6], 2, {1})
    run([10, 30, 20], [0, 2, 4, 6], 2, {1}, table=1)
    bad = torch.tensor([0, -5, 2, 3, 4, 5], dtype=torch.int32, device="cuda")
    run([10, 30, 20], [0, 2, 4, 6], 2, set(), pos=bad)


def test_own_stream(pkg):
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(10)
    s, counts, pos = shape(4, 2, 64), [20], np.arange(20)
    codes, exps = quantised(rng, 1, 64, 2, 64, 16)
    (q, k, v), (dq, dk, dv) = inputs(rng, s, counts, torch.bfloat16)
    got = []
    for side in (None, torch.cuda.Stream()):
        c = DeviceCache(pkg, {"k": codes, "v": codes.copy()}, {"k": exps, "v": exps.copy()}, [7], "slot")
        rows = device_rows(pkg, counts, pos)
        torch.cuda.synchronize()
        cc.cc_kv_append(s, c.cache, 0, rows, dk, dv, stream=side)
        assert cc.cc_get_status(side) == cc.CC_OK
        got.append((c.get("k"), c.get("k_exp")))
    np.testing.assert_array_equal(got[0][0], got[1][0])
    np.testing.assert_array_equal(got[0][1], got[1][1])
