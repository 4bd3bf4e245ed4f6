"""cc_kv_compact against the oracle (oracle/step.py), exactly: layouts, block sizes,
head counts and dims, keep-sets at the edges of blocks, chunks and pages, layers that are
missing, scales far apart and ones that are none; what lies past the kept slots; replays;
reports."""
import numpy as np
import pytest
import torch

import oracle
from tests._step import DeviceCache, quantised, shape

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    import paper_2607_27600_gb300 as p
    p.load_library()
    return p


class Case:
    """A cache of `layers` layers with everything that a slot carries, and its keep-set."""

    def __init__(self, pkg, seed, layers, hkv, dh, block, layout, cap, lens, keeps, stds=(0.02, 8.0), h=True,
                 page=128):
        rng = self.rng = np.random.default_rng(seed)
        self.pkg, self.block, self.lens, self.layout = pkg, block, lens, layout
        b = len(lens)
        self.s = shape(hkv * 2, hkv, dh)
        self.s = type(self.s)(**{**self.s.__dict__, "n_layers": layers, "d_model": 96})
        self.codes = [{n: None for n in "kv"} for _ in range(layers)]
        self.exps = [{n: None for n in "kv"} for _ in range(layers)]
        for l in range(layers):
            for n in "kv":
                c, e = quantised(rng, b, cap, hkv, dh, block, stds)
                for i, m in enumerate(lens):   # what lies past the ends may be anything
                    c[i, m:] = rng.integers(0, 256, c[i, m:].shape)
                    e[i, -(-m // block):] = rng.integers(0, 256, e[i, -(-m // block):].shape)
                self.codes[l][n], self.exps[l][n] = c, e
        self.small = {"tokens": rng.integers(0, 1000, (b, cap)).astype(np.int32),
                      "pos": rng.integers(0, 1 << 30, (b, cap)).astype(np.int32),
                      "h2o_acc": rng.standard_normal((b, cap)).astype(np.float32)}
        self.h = rng.integers(0, 1 << 15, (b, cap, 96)).astype(np.int16) if h else None
        self.keep = [np.sort(rng.choice(n, k, False)) if isinstance(k, int) else np.asarray(k)
                     for n, k in zip(lens, keeps)]
        self.page = page
        self.build()

    def build(self):
        c = self.c = DeviceCache(self.pkg, self.codes[0], self.exps[0], self.lens, self.layout, self.page)
        for n in "kv":
            c.d[n] = [c.put(x[n], c.page) if x[n] is not None else None for x in self.codes]
            c.d[n + "_exp"] = [c.put(x[n], c.page // self.block) if x[n] is not None else None for x in self.exps]
        for n, x in self.small.items():
            c.d[n] = torch.from_numpy(x.copy()).cuda()
        if self.h is not None:
            c.d["h_last"] = torch.from_numpy(self.h.copy()).cuda().view(torch.bfloat16)
        self.cache = self.pkg.Cache(c.d)
        self.count = torch.tensor([len(k) for k in self.keep], dtype=torch.int32, device="cuda")
        idx = self.rng.integers(-5, 1 << 20, (c.b, c.cap)).astype(np.int32)
        for i, k in enumerate(self.keep):
            idx[i, :len(k)] = k
        self.idx = torch.from_numpy(idx).cuda()

    def run(self, ws=None):
        from paper_2607_27600_gb300 import cc
        if ws is None:
            ws = cc.alloc_workspace(cc.cc_kv_compact_workspace_size(self.s, self.cache))
            ws.fill_(0xFF)
        cc.cc_kv_compact(self.s, self.cache, self.idx, self.count, ws)
        return cc.cc_get_status()

    def get(self, name, layer):
        """A layer's array as logical [B][n][...]."""
        return DeviceCache.get(self.at(layer), name)

    def at(self, layer):
        c = DeviceCache.__new__(DeviceCache)
        c.__dict__.update(self.c.__dict__)
        c.d = {n: [self.c.d[n][layer]] for n in ("k", "v", "k_exp", "v_exp")}
        return c

    def check(self, keep=None, but=None):
        """Everything, against the oracle; `but`: a sequence whose slots may hold anything."""
        keep = self.keep if keep is None else keep
        of = [i for i in range(len(self.lens)) if i != but]
        for l in range(len(self.codes)):
            for n in "kv":
                if self.codes[l][n] is None:
                    continue
                codes, exps = oracle.compact_blocks(self.codes[l][n], self.exps[l][n], self.block, keep)
                codes, exps, got = codes[of], exps[of], self.get(n, l)[of]
                nan = (got & 0x7F) == 0x7F
                np.testing.assert_array_equal(nan, (codes & 0x7F) == 0x7F)
                np.testing.assert_array_equal(np.where(nan, 0, got), np.where(nan, 0, codes))
                np.testing.assert_array_equal(self.get(n + "_exp", l)[of], exps)
        for n, x in self.small.items():
            want = x.copy()
            for i, k in enumerate(keep):
                want[i, :len(k)] = x[i, k]
            np.testing.assert_array_equal(self.c.d[n].cpu().numpy()[of], want[of])
        if self.h is not None:
            want = self.h.copy()
            for i, k in enumerate(keep):
                want[i, :len(k)] = self.h[i, k]
            np.testing.assert_array_equal(self.c.d["h_last"].view(torch.int16).cpu().numpy()[of], want[of])
        assert self.c.d["seq_len"].tolist() == [len(k) for k in keep]


CASES = [
    # layers, hkv, dh, block, layout, cap, lens, keeps
    (1, 1, 64, 16, "slot", 256, [1, 0, 17, 256, 255], [1, 0, 16, 256, 129]),
    (2, 2, 64, 32, "paged", 512, [512, 300, 129, 128], [100, 299, 128, 1]),
    (2, 3, 64, 16, "slot", 384, [384, 383, 200], [127, 128, 33]),             # an odd head of 64
    (3, 8, 128, 64, "head", 640, [640, 513, 64, 0], [600, 512, 63, 0]),
    (1, 4, 128, 128, "paged", 1024, [1024, 900, 128], [1023, 130, 100]),
    (2, 5, 128, 16, "slot", 144, [144, 130, 16], [143, 40, 15]),              # a cap of no whole chunks
    (1, 2, 64, 128, "head", 2048, [2048, 1500], [2040, 1]),
    (4, 1, 128, 32, "paged", 4096, [4000, 4096, 5], [1000, 4001, 5]),
]


@pytest.mark.parametrize("layers,hkv,dh,block,layout,cap,lens,keeps", CASES)
def test_matches_oracle(pkg, layers, hkv, dh, block, layout, cap, lens, keeps):
    from paper_2607_27600_gb300 import cc
    c = Case(pkg, hkv * 1000 + cap, layers, hkv, dh, block, layout, cap, lens, keeps)
    assert c.run() == cc.CC_OK
    c.check()


@pytest.mark.parametrize("layout", ["slot", "paged", "head"])
def test_keep_sets(pkg, layout):
    """All, none, the first ones, all but the first, the last ones, every other one, one from each
    chunk, and from a chunk's first half."""
    from paper_2607_27600_gb300 import cc
    n = 768
    keep = [range(n), [], range(400), range(1, n), range(500, n), range(0, n, 2), range(77, n, 128),
            [i for i in range(n) if i % 128 < 64]]
    c = Case(pkg, 5, 2, 2, 64, 16, layout, n, [n] * len(keep), [np.asarray(list(k), int) for k in keep])
    assert c.run() == cc.CC_OK
    c.check()


@pytest.mark.parametrize("block", [16, 64, 128])
def test_scales_far_apart(pkg, block):
    """Exponents from one end to the other, 0 and 255 among them: falls of every size."""
    from paper_2607_27600_gb300 import cc
    c = Case(pkg, 6, 1, 2, 128, block, "paged", 2048, [2048, 2000], [700, 650])
    for n in "kv":
        near = 100 + c.rng.integers(-25, 25, c.exps[0][n].shape)
        far = c.rng.integers(0, 256, c.exps[0][n].shape)
        c.exps[0][n] = np.where(c.rng.random(near.shape) < 0.15, far, near).astype(np.uint8)
        c.codes[0][n] = c.rng.integers(0, 256, c.codes[0][n].shape).astype(np.uint8)
    c.build()
    assert c.run() == cc.CC_OK
    c.check()


def test_every_code_and_fall(pkg):
    """Each of the 256 codes at a scale 0 to 31 steps below its block's, to nearest, ties to even."""
    from paper_2607_27600_gb300 import cc
    falls, dh = 32, 128
    # blocks of 16 slots: even blocks at 120, of which one slot is kept; odd ones lower
    c = Case(pkg, 7, 1, 1, dh, 16, "slot", 2 * falls * 16, [2 * falls * 16], [1], h=False)
    keep = []
    for f in range(falls):
        c.exps[0]["k"][0, 2 * f], c.exps[0]["k"][0, 2 * f + 1] = 120, 120 - f
        for half in range(2):
            c.codes[0]["k"][0, (2 * f + 1) * 16 + half, 0] = np.arange(half * dh, (half + 1) * dh)
        # a new block: 14 slots of the higher scale, then the two halves of the codes
        keep += [2 * f * 16 + i for i in range(14)] + [(2 * f + 1) * 16, (2 * f + 1) * 16 + 1]
    c.keep = [np.asarray(keep)]
    c.build()
    assert c.run() == cc.CC_OK
    c.check()


def test_missing_arrays(pkg):
    """Layers without K and V, a cache without totals or H."""
    from paper_2607_27600_gb300 import cc
    c = Case(pkg, 8, 3, 2, 64, 32, "slot", 256, [200, 256], [50, 60], h=False)
    c.codes[1] = c.exps[1] = {"k": None, "v": None}
    del c.small["h2o_acc"]
    c.build()
    assert c.run() == cc.CC_OK
    c.check()


def test_repeated_and_replayed(pkg):
    """Refresh after refresh, recorded once and replayed: counts and keep-sets are read
    at each replay."""
    from paper_2607_27600_gb300 import cc
    c = Case(pkg, 9, 2, 2, 64, 16, "paged", 1024, [1000, 512], [700, 300])
    ws = cc.alloc_workspace(cc.cc_kv_compact_workspace_size(c.s, c.cache))
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    cc.cc_kv_compact(c.s, c.cache, c.idx, c.count, ws, stream=st)
    assert cc.cc_get_status(st) == cc.CC_OK
    c.check()
    cc.cc_graph_begin(st)
    cc.cc_kv_compact(c.s, c.cache, c.idx, c.count, ws, stream=st)
    g = cc.cc_graph_end(st)
    try:
        for n0, n1 in ((400, 299), (399, 1), (50, 1)):
            c.codes = [{n: c.get(n, l).astype(np.uint8) for n in "kv"} for l in range(2)]
            c.exps = [{n: c.get(n + "_exp", l).astype(np.uint8) for n in "kv"} for l in range(2)]
            c.small = {n: c.c.d[n].cpu().numpy() for n in c.small}
            c.h = c.c.d["h_last"].view(torch.int16).cpu().numpy()
            c.keep = [np.sort(c.rng.choice(len(k), n, False)) for k, n in zip(c.keep, (n0, n1))]
            for i, k in enumerate(c.keep):
                c.idx[i, :len(k)] = torch.from_numpy(k.astype(np.int32)).cuda()
            c.count.copy_(torch.tensor([n0, n1]))
            st.wait_stream(torch.cuda.current_stream())
            cc.cc_graph_launch(g, st)
            assert cc.cc_get_status(st) == cc.CC_OK
            c.check()
    finally:
        cc.cc_graph_destroy(g)


def test_bad_keep_sets_are_reported(pkg):
    """A count that is none leaves its sequence's slots (length 0); an entry out of order or
    range, or the same twice, leaves the other sequences' results."""
    from paper_2607_27600_gb300 import cc
    c = Case(pkg, 10, 1, 2, 64, 16, "slot", 512, [500, 500, 512], [100, 200, 300])
    c.count[1] = 513
    assert c.run() == cc.CC_ERR_DEVICE_ARG
    c.check([c.keep[0], [], c.keep[2]])
    for bad in (3, 512, -1, 505, None):
        c = Case(pkg, 10, 1, 2, 64, 16, "slot", 512, [500, 500, 512], [100, 200, 300])
        c.idx[1, 199 if bad == 505 else 64] = int(c.idx[1, 63]) if bad is None else bad
        assert c.run() == cc.CC_ERR_DEVICE_ARG, bad
        c.check(but=1)


def test_pages_that_are_none(pkg):
    """A source's page outside the pool leaves its slots out, a destination's too."""
    from paper_2607_27600_gb300 import cc
    c = Case(pkg, 12, 1, 2, 64, 16, "paged", 512, [512, 512], [range(0, 512, 2), 200], h=False)
    before = c.get("k", 0)
    c.c.d["block_table"][0, 2] = -1
    assert c.run() == cc.CC_ERR_DEVICE_ARG
    got = c.get("k", 0)
    # slots 128 to 191 come from the page that is not there
    np.testing.assert_array_equal(got[0, 128:192], before[0, 128:192])
    codes, _ = oracle.compact_blocks(c.codes[0]["k"], c.exps[0]["k"], 16, c.keep)
    np.testing.assert_array_equal(got[0, :128], codes[0, :128])
    np.testing.assert_array_equal(got[0, 192:256], codes[0, 192:256])
    np.testing.assert_array_equal(got[1], codes[1])


def test_many_sequences(pkg):
    """More sequences than the first chunks in shared memory, most of them short."""
    from paper_2607_27600_gb300 import cc
    b = 1030
    rng = np.random.default_rng(13)
    lens = rng.integers(0, 129, b).tolist()
    c = Case(pkg, 13, 1, 1, 64, 32, "slot", 128, lens, [int(rng.integers(0, n + 1)) for n in lens], h=False)
    assert c.run() == cc.CC_OK
    c.check()


def test_refusals(pkg):
    from paper_2607_27600_gb300 import cc
    c = Case(pkg, 14, 1, 2, 64, 16, "slot", 256, [100], [50])
    ws = cc.alloc_workspace(cc.cc_kv_compact_workspace_size(c.s, c.cache))
    for idx, count in ((c.idx[:, :-1], c.count), (c.idx.long(), c.count), (c.idx, c.count.long()),
                       (c.idx, c.idx[0, :2])):
        with pytest.raises(ValueError):
            cc.cc_kv_compact(c.s, c.cache, idx, count, ws)
    with pytest.raises(cc.CCError):
        cc.cc_kv_compact(c.s, c.cache, c.idx, c.count, ws[:16])
    assert torch.equal(c.c.d["seq_len"], torch.tensor([100], dtype=torch.int32, device="cuda"))
