"""cc_kv_accumulate against the fp64 oracle (oracle/step.py): head groups and dims,
layouts, block sizes, row counts from one token to chunks, lengths at the edges of
tiles, blocks and pages, sequences without rows or slots, rows without a finite lse,
scales that are none, strides and what lies past the ends; reports.

Tolerances.  A weight is 2^(x - y), x a product of head_dim fp32 terms (exact operands)
times a factor, y the row's lse.  Eight or fewer product instructions add to x, each with
a truncation or two of the sum so far: 2^-19 of A = sum_i |q_i K_i| / sqrt(head_dim); the factors'
roundings: 2^-22 of |x| and |y|.  The exponential: 2^-21.  A slot's sum of N terms:
N 2^-24 of it, and its total 2^-24 once per pass."""
import numpy as np
import pytest
import torch

import oracle
from tests._step import DeviceCache, columns, device_rows, quantised, shape, starts, values

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def pkg():
    import paper_2607_27600_gb300 as p
    p.load_library()
    return p


class Case:
    """A cache with totals, rows with their lse (from the oracle), on both sides."""

    def __init__(self, pkg, seed, hq, hkv, dh, block, layout, dtype, cap, lens, counts, memory=False, stds=(0.5, 2.0)):
        rng = self.rng = np.random.default_rng(seed)
        self.pkg, self.s, self.lens, self.counts, self.memory = pkg, shape(hq, hkv, dh), lens, counts, memory
        self.codes, self.exps = {}, {}
        for n in "kv":
            self.codes[n], self.exps[n] = quantised(rng, len(lens), cap, hkv, dh, block, stds)
        self.ends = [n + (0 if memory or not m else m) for n, m in zip(lens, counts)]
        for i, n in enumerate(self.ends):   # NaN codes and any exponents past the ends
            self.codes["k"][i, n:] = 0x7F
            self.exps["k"][i, -(-n // block):] = rng.integers(0, 256, self.exps["k"][i, -(-n // block):].shape)
        self.t = TYPES[dtype]
        self.q = torch.from_numpy(rng.standard_normal((sum(counts), hq, dh)) * 1.5).to(self.t).double().numpy()
        self.k = values(self.codes["k"], self.exps["k"])
        self.start = starts(counts)
        _, lse, _ = oracle.attend_rows(self.q, self.k, self.k * 0, lens, self.start, memory)
        self.lse = lse.astype(np.float32)
        self.acc = rng.uniform(0, 2, (len(lens), cap)).astype(np.float32)
        self.c = DeviceCache(pkg, self.codes, self.exps, lens, layout)

    def run(self, first=False, pad=24):
        from paper_2607_27600_gb300 import cc
        dq, = columns([self.q], self.t, pad)
        acc = torch.from_numpy(self.acc).cuda()
        cache = self.pkg.Cache({**self.c.d, "h2o_acc": acc})
        rows = device_rows(self.pkg, self.counts)
        ws = cc.alloc_workspace(cc.cc_kv_accumulate_workspace_size(self.s, cache, rows))
        ws.fill_(0xFF)
        cc.cc_kv_accumulate(self.s, cache, 0, rows, dq, torch.from_numpy(self.lse).cuda(), ws, first=first,
                            memory_only=self.memory)
        return acc.cpu().numpy()

    def want(self, first=False):
        base = self.acc.astype(np.float64)
        if first:
            for i, (n, m) in enumerate(zip(self.lens, self.counts)):
                base[i, n:n + m] = 0
        got, slack = oracle.received(self.q, self.k, self.lse, self.lens, self.start, self.memory)
        terms = max(self.counts) * self.s.n_q_heads
        return base + got, 2.0 ** -19 * slack + (terms * 2.0 ** -24 + 2.0 ** -20) * got + 2.0 ** -22 * (base + got)

    def check(self, got, first=False):
        want, tol = self.want(first)
        off = np.abs(got - want) / np.maximum(tol, 1e-30)
        at = np.unravel_index(np.where(np.isnan(off), np.inf, off).argmax(), off.shape)
        assert off[at] <= 1, (at, got[at], want[at], tol[at])
        for i, n in enumerate(self.ends):   # slots that no row sees: untouched
            np.testing.assert_array_equal(got[i, n if self.counts[i] else 0:], self.acc[i, n if self.counts[i] else 0:])


EDGES = [0, 1, 14, 15, 16, 17, 62, 63, 64, 65, 126, 127, 128, 190, 254]
CASES = [
    # hq, hkv, dh, block, layout, dtype, cap, lens, counts
    (1, 1, 64, 16, "slot", "bf16", 256, EDGES, [1] * 15),
    (8, 2, 64, 128, "paged", "f16", 256, EDGES, [1] * 15),
    (7, 1, 128, 32, "head", "bf16", 256, EDGES, [1] * 15),
    (5, 5, 128, 64, "slot", "f16", 256, EDGES, [1] * 15),
    (16, 2, 128, 64, "paged", "bf16", 256, EDGES, [1] * 15),
    (72, 1, 64, 16, "paged", "bf16", 128, [0, 100], [1, 1]),             # nine eights of rows
    (8, 2, 128, 16, "paged", "f16", 256, [0, 3, 250, 100, 77], [4, 0, 6, 3, 5]),
    (8, 8, 64, 64, "paged", "bf16", 1024, [1000, 1, 0], [24, 16, 9]),
    (64, 64, 128, 32, "slot", "bf16", 128, [90, 17], [2, 1]),            # more heads than a pass holds
    (4, 4, 128, 64, "slot", "bf16", 2560, [2500, 2501, 9], [1, 1, 1]),
    (8, 1, 64, 16, "paged", "f16", 4096, [4000, 17], [1, 1]),
    (14, 2, 64, 32, "head", "f16", 384, [300, 0, 60], [12, 40, 3]),
]


@pytest.mark.parametrize("memory", [False, True])
@pytest.mark.parametrize("hq,hkv,dh,block,layout,dtype,cap,lens,counts", CASES)
def test_matches_oracle(pkg, hq, hkv, dh, block, layout, dtype, cap, lens, counts, memory):
    from paper_2607_27600_gb300 import cc
    c = Case(pkg, hq * 1000 + cap, hq, hkv, dh, block, layout, dtype, cap, lens, counts, memory)
    got = c.run()
    assert cc.cc_get_status() == cc.CC_OK
    c.check(got)
    np.testing.assert_array_equal(c.run(), got)   # the same bits, run to run


CHUNKS = [
    (8, 2, 64, 16, "paged", 512, [0, 130, 300], [200, 150, 64]),
    (4, 1, 128, 64, "head", 1024, [777], [130]),
    (7, 1, 128, 128, "slot", 384, [0, 1, 127, 128], [257, 64, 128, 129]),
    (16, 2, 64, 32, "paged", 256, [10, 0, 90, 256], [100, 40, 0, 0]),
    (3, 3, 128, 32, "paged", 2304, [2048], [72]),
    (6, 2, 128, 16, "slot", 768, [511, 1, 0], [129, 255, 1]),
]


@pytest.mark.parametrize("memory", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,dh,block,layout,cap,lens,counts", CHUNKS)
def test_chunks_match_oracle(pkg, hq, hkv, dh, block, layout, cap, lens, counts, dtype, memory):
    from paper_2607_27600_gb300 import cc
    c = Case(pkg, hq * 1000 + cap, hq, hkv, dh, block, layout, dtype, cap, lens, counts, memory)
    got = c.run()
    assert cc.cc_get_status() == cc.CC_OK
    c.check(got)
    np.testing.assert_array_equal(c.run(), got)


WIDE = [
    # groups of many heads: a tile of one or two positions, and more than a tile holds
    (96, 1, 64, 16, "paged", 256, [50, 130], [70, 2]),
    (56, 1, 128, 64, "slot", 384, [301], [33]),
    (48, 1, 64, 32, "head", 256, [0, 200], [41, 5]),
    (128, 1, 64, 16, "slot", 256, [100, 3], [40, 1]),
    (256, 1, 128, 32, "head", 256, [30, 77], [5, 0]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,dh,block,layout,cap,lens,counts", WIDE)
def test_wide_groups(pkg, hq, hkv, dh, block, layout, cap, lens, counts, dtype):
    from paper_2607_27600_gb300 import cc
    c = Case(pkg, hq * 1000 + cap, hq, hkv, dh, block, layout, dtype, cap, lens, counts, False)
    got = c.run()
    assert cc.cc_get_status() == cc.CC_OK
    c.check(got)
    np.testing.assert_array_equal(c.run(), got)


@pytest.mark.parametrize("memory", [False, True])
@pytest.mark.parametrize("most", [3, 90])
def test_many_sequences(pkg, most, memory):
    """More sequences than a warp has lanes, some without slots, some without rows."""
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(most)
    lens, counts = rng.integers(0, 160, 70), rng.integers(0, most + 1, 70)
    lens[rng.integers(0, 70, 20)] = 0
    counts[rng.integers(0, 70, 20)] = 0
    c = Case(pkg, most, 8, 2, 64, 32, "paged", "bf16", 256, [int(x) for x in lens], [int(x) for x in counts], memory)
    got = c.run()
    assert cc.cc_get_status() == cc.CC_OK
    c.check(got)
    np.testing.assert_array_equal(c.run(), got)


@pytest.mark.parametrize("counts", [[1, 1, 1], [100, 3, 64]])
def test_first_layer_of_a_step(pkg, counts):
    """The rows' own slots start from 0, whatever they held."""
    c = Case(pkg, 3, 8, 2, 64, 32, "paged", "bf16", 512, [37, 0, 128], counts)
    for i, (n, m) in enumerate(zip(c.lens, counts)):
        c.acc[i, n:n + m] = np.nan
    got = c.run(first=True)
    c.acc = np.nan_to_num(c.acc)
    c.check(got, first=True)


@pytest.mark.parametrize("counts", [[1, 5], [150, 40]])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_rows_without_a_finite_lse_add_nothing(pkg, counts, dtype):
    """Even where their slots or their queries are no numbers."""
    c = Case(pkg, 4, 8, 2, 64, 16, "slot", dtype, 512, [200, 33], counts)
    whole = c.run()
    # every row of sequence 0 sees a slot of KV head 0 that is no number: its attention had no lse
    c.codes["k"][0, 20, 0, 3] = 0x7F
    c.lse[:counts[0], :4] = np.nan
    c.q[0, 1] = np.inf
    c.lse[counts[0]:, 6] = -np.inf
    c.lse[-1, 7] = np.inf
    c.k = values(c.codes["k"], c.exps["k"])
    c.c = DeviceCache(c.pkg, c.codes, c.exps, c.lens, "slot")
    got = c.run()
    c.check(got)
    assert (got[:, :30] < whole[:, :30]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("counts", [[1], [130]])
def test_every_code(pkg, counts, dtype):
    """All codes that are numbers, the least ones under a scale that makes them count."""
    c = Case(pkg, 9, 4, 1, 128, 16, "slot", dtype, 512, [320], counts)
    numbers = np.array([x for x in range(256) if x & 0x7F != 0x7F], np.uint8)
    c.codes["k"][0, :, 0] = c.rng.choice(numbers, c.codes["k"][0, :, 0].shape)
    c.codes["k"][0, :160, 0] &= 0x87          # subnormal ones
    c.exps["k"][:] = 118
    c.exps["k"][0, :10] = 132
    c.k = values(c.codes["k"], c.exps["k"])
    _, lse, _ = oracle.attend_rows(c.q, c.k, c.k * 0, c.lens, c.start)
    c.lse = lse.astype(np.float32)
    c.c = DeviceCache(c.pkg, c.codes, c.exps, c.lens, "slot")
    c.check(c.run())


def test_not_a_number_under_a_finite_lse(pkg):
    """A slot that is no number with an lse that knows nothing of it: its total is NaN, no other."""
    for counts in ([1], [130]):
        for dtype in TYPES:
            c = Case(pkg, 10, 4, 2, 64, 16, "slot", dtype, 256, [100], counts)
            c.codes["k"][0, 20, 1, 5] = 0xFF
            c.c = DeviceCache(c.pkg, c.codes, c.exps, c.lens, "slot")
            got = c.run()
            assert np.isnan(got[0, 20])
            got[0, 20] = c.want()[0][0, 20]
            c.check(got)


def test_scales_that_are_none(pkg):
    """An exponent of 0 makes scores of 0; rows that see one of 255 come without an lse."""
    c = Case(pkg, 5, 4, 2, 128, 16, "paged", "bf16", 256, [100, 60], [1, 3])
    c.exps["k"][0, 2], c.exps["k"][1, 1] = 0, 255
    c.k = values(c.codes["k"], c.exps["k"])
    c.k[0, 32:48] = 0
    c.k[1, 16:32] = 0
    _, lse, _ = oracle.attend_rows(c.q, c.k, c.k * 0, c.lens, c.start)
    c.lse = lse.astype(np.float32)
    c.lse[1:] = np.nan
    c.c = DeviceCache(c.pkg, c.codes, c.exps, c.lens, "paged")
    c.check(c.run())


@pytest.mark.parametrize("counts", [[1, 1], [80, 150]])
def test_scales_and_scores_far_apart(pkg, counts):
    """Scores of hundreds, whose weights go from 1 to nothing."""
    c = Case(pkg, 6, 8, 2, 64, 16, "slot", "bf16", 512, [300, 222], counts, stds=(0.01, 60.0))
    c.check(c.run())


@pytest.mark.parametrize("counts", [[1, 1, 1], [70, 90, 110]])
def test_bad_sequences_are_reported_and_skipped(pkg, counts):
    from paper_2607_27600_gb300 import cc
    c = Case(pkg, 7, 8, 2, 64, 16, "paged", "bf16", 256, [100, 50, 140], counts)
    good = c.run()
    c.c.d["seq_len"][1] = 257
    got = c.run()
    assert cc.cc_get_status() == cc.CC_ERR_DEVICE_ARG
    np.testing.assert_array_equal(got[[0, 2]], good[[0, 2]])
    np.testing.assert_array_equal(got[1], c.acc[1])
    c.c.d["seq_len"][1] = 50
    c.c.d["block_table"][2, 0] = c.c.n_pages   # a page that is none: its slots receive nothing
    got = c.run()
    assert cc.cc_get_status() == cc.CC_ERR_DEVICE_ARG
    np.testing.assert_array_equal(got[:2], good[:2])
    np.testing.assert_array_equal(got[2, :128], c.acc[2, :128])
    np.testing.assert_array_equal(got[2, 128:], good[2, 128:])


def test_refusals(pkg):
    from paper_2607_27600_gb300 import cc
    c = Case(pkg, 8, 8, 2, 64, 16, "slot", "bf16", 256, [100], [1])
    acc = torch.zeros(1, 256, device="cuda")
    cache = pkg.Cache({**c.c.d, "h2o_acc": acc})
    rows, ws = device_rows(pkg, [1]), cc.alloc_workspace(1 << 20)
    q, lse = torch.zeros(1, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 8, device="cuda")
    for bad in (dict(q=q[:, :4]), dict(q=q.double()), dict(lse=lse[:, :4]), dict(lse=lse.half())):
        with pytest.raises(ValueError):
            cc.cc_kv_accumulate(c.s, cache, 0, rows, **{"q": q, "lse": lse, "ws": ws, **bad})
    for bad in (dict(q=q.float()), dict(first=True, memory_only=True), dict(ws=ws[:16])):
        with pytest.raises(cc.CCError):
            cc.cc_kv_accumulate(c.s, cache, 0, rows, **{"q": q, "lse": lse, "ws": ws, **bad})
    with pytest.raises(cc.CCError):
        cc.cc_kv_accumulate(c.s, c.c.cache, 0, rows, q, lse, ws)   # no totals in the cache
