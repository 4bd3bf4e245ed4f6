"""The cache's management as a serving loop uses it: a batch whose sequences share a prefix
that is held once, attention over it and over each sequence's own memory joined, totals
of what every slot receives, a refresh by them, and on; eagerly and replayed from
graphs that share a workspace, on a stream of its own; offsets past 32 bits."""
import math

import numpy as np
import pytest
import torch

import oracle
from synth.configs import ModelShape
from tests._step import shape, starts, values

pytestmark = pytest.mark.gpu
LAYERS, HQ, HKV, DH, BLOCK, CAP, PREFIX = 2, 8, 2, 64, 16, 256, 150


@pytest.fixture(scope="module")
def pkg():
    import paper_2607_27600_gb300 as p
    p.load_library()
    return p


def empty_cache(pkg, batch, cap):
    def zeros(*dims):
        return [torch.zeros(dims, dtype=torch.uint8, device="cuda") for _ in range(LAYERS)]
    return pkg.Cache({"k": zeros(batch, cap, HKV, DH), "v": zeros(batch, cap, HKV, DH),
                      "k_exp": zeros(batch, cap // BLOCK, HKV), "v_exp": zeros(batch, cap // BLOCK, HKV),
                      "kv_block": BLOCK, "seq_len": torch.zeros(batch, dtype=torch.int32, device="cuda"),
                      "tokens": torch.zeros(batch, cap, dtype=torch.int32, device="cuda"),
                      "pos": torch.zeros(batch, cap, dtype=torch.int32, device="cuda"),
                      "h2o_acc": torch.full((batch, cap), float("nan"), device="cuda")})


def logical(cache, layer, name):
    return values(cache.d[name][layer].cpu().numpy(), cache.d[name + "_exp"][layer].cpu().numpy())


class Loop:
    """Three sequences over one prefix; the rows' projections are random."""

    def __init__(self, pkg, seed=0):
        from paper_2607_27600_gb300 import cc
        self.pkg, self.cc = pkg, cc
        s = shape(HQ, HKV, DH)
        self.s = ModelShape(**{**s.__dict__, "n_layers": LAYERS})
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.prefix, self.own = empty_cache(pkg, 1, 256), empty_cache(pkg, 3, CAP)
        rows = pkg.Rows(PREFIX, torch.tensor([0, PREFIX], dtype=torch.int32, device="cuda"), None, PREFIX)
        for l in range(LAYERS):
            x = self.draw(PREFIX)
            cc.cc_kv_append(self.s, self.prefix, l, rows, x[:, HQ:HQ + HKV], x[:, HQ + HKV:])
        cc.cc_kv_advance(self.prefix, rows)
        self.prefix.d["h2o_acc"].zero_()

    def draw(self, n):
        return torch.randn(n, HQ + 2 * HKV, DH, generator=self.g, device="cuda").to(torch.bfloat16)

    def buffers(self, counts):
        n = sum(counts)
        b = type("Buffers", (), {})()
        b.counts = counts
        b.x = torch.empty(LAYERS, n, HQ + 2 * HKV, DH, dtype=torch.bfloat16, device="cuda")
        b.pos = torch.zeros(n, dtype=torch.int32, device="cuda")
        b.rows = self.pkg.Rows(n, torch.from_numpy(starts(counts)).cuda(), b.pos, max(counts))
        # over the prefix the rows are those of one sequence
        b.flat = self.pkg.Rows(n, torch.tensor([0, n], dtype=torch.int32, device="cuda"), b.pos, n)
        b.q = [torch.empty(n, HQ, DH, dtype=torch.bfloat16, device="cuda") for _ in range(LAYERS)]
        b.part = torch.empty(2, n, HQ, DH, dtype=torch.bfloat16, device="cuda")
        b.part_lse = torch.empty(2, n, HQ, device="cuda")
        b.out = torch.empty(LAYERS, n, HQ, DH, dtype=torch.bfloat16, device="cuda")
        b.lse = torch.empty(LAYERS, n, HQ, device="cuda")
        return b

    def workspace(self, *buffers):
        cc = self.cc
        return cc.alloc_workspace(max(f(self.s, c, r) for b in buffers for c, r in ((self.prefix, b.flat), (self.own, b.rows))
                                      for f in (cc.cc_kv_attention_workspace_size, cc.cc_kv_accumulate_workspace_size)))

    def step(self, b, ws, stream=None):
        cc, s = self.cc, self.s
        for l in range(LAYERS):
            x = b.x[l]
            cc.cc_kv_append(s, self.own, l, b.rows, x[:, HQ:HQ + HKV], x[:, HQ + HKV:], x[:, :HQ], b.q[l], stream=stream)
            cc.cc_kv_attention(s, self.prefix, l, b.flat, b.q[l], b.part[0], ws, lse=b.part_lse[0], memory_only=True,
                               stream=stream)
            cc.cc_kv_attention(s, self.own, l, b.rows, b.q[l], b.part[1], ws, lse=b.part_lse[1], stream=stream)
            cc.cc_kv_join(s, list(b.part), list(b.part_lse), b.out[l], b.lse[l], stream=stream)
            cc.cc_kv_accumulate(s, self.own, l, b.rows, b.q[l], b.lse[l], ws, first=l == 0, stream=stream)
            cc.cc_kv_accumulate(s, self.prefix, l, b.flat, b.q[l], b.lse[l], ws, memory_only=True, stream=stream)
        cc.cc_kv_advance(self.own, b.rows, stream=stream)

    def feed(self, b):
        b.x.copy_(torch.stack([self.draw(len(b.pos)) for _ in range(LAYERS)]))
        lens = self.own.d["seq_len"].tolist()
        b.pos.copy_(torch.cat([torch.arange(PREFIX + 7 * i + n, PREFIX + 7 * i + n + m) for i, (n, m) in
                               enumerate(zip(lens, b.counts))]).to(torch.int32))
        return lens

    def check(self, b, lens, before):
        """The step's rows over prefix and own memory as one cache, in 64 bits; the totals it added."""
        start = starts(b.counts)
        own = before["own"].copy()
        for i, (n, m) in enumerate(zip(lens, b.counts)):
            own[i, n:n + m] = 0
        want_own, want_prefix, tol_own, tol_prefix = own, before["prefix"].copy(), np.abs(own) * 0, np.abs(before["prefix"]) * 0
        for l in range(LAYERS):
            q, lse = b.q[l].double().cpu().numpy(), b.lse[l].double().cpu().numpy()
            pk, pv = (np.repeat(logical(self.prefix, l, n)[:, :PREFIX], 3, 0) for n in "kv")
            ok, ov = (logical(self.own, l, n) for n in "kv")
            both = [np.concatenate([a, x], 1) for a, x in ((pk, ok), (pv, ov))]
            want, want_lse, spread = oracle.attend_rows(q, *both, [PREFIX + n for n in lens], start)
            got = b.out[l].double().cpu().numpy()
            # two parts and their join are rounded to bf16 (2^-8 each time), each part's probabilities too
            # where they are tiles (2^-8, and as much for their scores)
            assert (np.abs(got - want) <= (2 * 2.0 ** -8 + 2 * 2.0 ** -8) * spread).all()
            assert (np.abs(lse - want_lse) <= 2.0 ** -11 + 2.0 ** -21 * np.abs(want_lse)).all()
            for cache, k, ln, st, memory, total, tol in (
                    (self.own, ok, lens, start, False, want_own, tol_own),
                    (self.prefix, pk[:1], [PREFIX], [0, len(q)], True, want_prefix, tol_prefix)):
                add, slack = oracle.received(q, k, lse, ln, st, memory)
                total[:, :add.shape[1]] += add
                tol[:, :add.shape[1]] += 2.0 ** -19 * slack + 2.0 ** -14 * add
        for cache, total, tol in ((self.own, want_own, tol_own), (self.prefix, want_prefix, tol_prefix)):
            got = cache.d["h2o_acc"].double().cpu().numpy()
            for i, n in enumerate(cache.d["seq_len"].tolist()):
                assert (np.abs(got[i, :n] - total[i, :n]) <= tol[i, :n] + 2.0 ** -21 * np.abs(total[i, :n])).all()

    def totals(self):
        return {n: np.nan_to_num(c.d["h2o_acc"].double().cpu().numpy()) for n, c in (("own", self.own), ("prefix", self.prefix))}

    def refresh(self, budget, recent, stream=None):
        """Down to `budget` slots a sequence, the most recent among them; the keep-sets."""
        cc, d = self.cc, self.own.d
        lens = d["seq_len"].tolist()
        scores = torch.empty(3, CAP, device="cuda")
        idx = torch.empty(3, CAP, dtype=torch.int32, device="cuda")
        count = torch.empty(3, dtype=torch.int32, device="cuda")
        cc.cc_score_h2o(self.own, recent, scores, stream=stream)
        cc.cc_select_keep(scores, d["seq_len"], 3, CAP, torch.full((3,), budget, dtype=torch.int32, device="cuda"), 0,
                          idx, count, stream=stream)
        acc = d["h2o_acc"].cpu().numpy().copy()
        old = {n: [x.cpu().numpy().copy() for x in d[n]] for n in ("k", "v", "k_exp", "v_exp")}
        ws = cc.alloc_workspace(cc.cc_kv_compact_workspace_size(self.s, self.own))
        cc.cc_kv_compact(self.s, self.own, idx, count, ws, stream=stream)
        assert cc.cc_get_status(stream) == cc.CC_OK
        keep = []
        for i, n in enumerate(lens):
            j = min(budget, n)
            recents = np.arange(max(0, n - recent), n)
            rest = np.lexsort((-np.arange(n - len(recents)), -acc[i, :n - len(recents)]))[:max(0, j - len(recents))]
            want = np.sort(np.concatenate([rest, recents]))[-j:]
            assert int(count[i]) == j
            np.testing.assert_array_equal(idx[i, :j].cpu().numpy(), want)
            np.testing.assert_array_equal(d["h2o_acc"][i, :j].cpu().numpy(), acc[i, want])
            keep.append(want)
        assert d["seq_len"].tolist() == [len(k) for k in keep]
        for l in range(LAYERS):
            for n in "kv":
                codes, exps = oracle.compact_blocks(old[n][l], old[n + "_exp"][l], BLOCK, keep)
                np.testing.assert_array_equal(d[n][l].cpu().numpy(), codes)
                np.testing.assert_array_equal(d[n + "_exp"][l].cpu().numpy(), exps)


def test_a_loop_with_a_shared_prefix(pkg):
    """Prompts as chunks, single tokens, a refresh, and on; every step against 64 bits."""
    loop = Loop(pkg)
    prompts, one, few = loop.buffers([90, 0, 33]), loop.buffers([1, 1, 1]), loop.buffers([3, 1, 5])
    ws = loop.workspace(prompts, one, few)
    for b in (prompts, one, few, one):
        before, lens = loop.totals(), loop.feed(b)
        loop.step(b, ws)
        assert loop.cc.cc_get_status() == loop.cc.CC_OK
        loop.check(b, lens, before)
    loop.refresh(24, 4)
    for b in (one, prompts, one):
        before, lens = loop.totals(), loop.feed(b)
        loop.step(b, ws)
        assert loop.cc.cc_get_status() == loop.cc.CC_OK
        loop.check(b, lens, before)
    loop.refresh(60, 8)


def test_replayed_on_a_stream_of_its_own(pkg):
    """Two recorded steps that share a workspace, replayed by turns around a refresh: the bits of eager steps."""
    ends = []
    for captured in (False, True):
        loop = Loop(pkg, seed=1)
        cc, side = loop.cc, torch.cuda.Stream()
        prompts, one = loop.buffers([70, 20, 5]), loop.buffers([1, 1, 1])
        ws = loop.workspace(prompts, one)
        side.wait_stream(torch.cuda.current_stream())
        graphs = {}
        if captured:
            for name, b in (("prompts", prompts), ("one", one)):
                cc.cc_graph_begin(side)
                loop.step(b, ws, side)
                graphs[name] = cc.cc_graph_end(side)
        outs = []
        for name in ("prompts", "one", "one", "refresh", "one", "prompts", "one"):
            torch.cuda.synchronize()
            if name == "refresh":
                loop.refresh(30, 4, side)
                continue
            b = prompts if name == "prompts" else one
            loop.feed(b)
            torch.cuda.synchronize()
            if captured:
                cc.cc_graph_launch(graphs[name], side)
            else:
                loop.step(b, ws, side)
            torch.cuda.synchronize()
            outs += [b.out.clone(), b.lse.clone()]
        assert cc.cc_get_status(side) == cc.CC_OK
        for g in graphs.values():
            cc.cc_graph_destroy(g)
        n = loop.own.d["seq_len"].tolist()
        assert n == [102, 44, 14]   # 72, 22 and 7 slots, of which 30, 22 and 7 are kept; then 1 + prompts + 1
        ends.append(outs + [loop.own.d["h2o_acc"][i, :m] for i, m in enumerate(n)] + [loop.prefix.d["h2o_acc"]]
                    + loop.own.d["k"] + loop.own.d["v_exp"])
    for a, b in zip(*ends):
        assert torch.equal(a, b)


def test_offsets_past_32_bits(pkg):
    """Slots at the end of buffers of 4.6 GB: what they receive from single rows and from a chunk, and a
    refresh that keeps some of them, as if the buffers were small."""
    from paper_2607_27600_gb300 import cc
    hkv, dh, block, cap, tail = 32, 128, 128, 1130496, 300
    assert cap * hkv * dh > 2 ** 32 and cap % 128 == 0
    s = shape(hkv, hkv, dh)
    g = torch.Generator(device="cuda").manual_seed(5)
    for layout in ("slot", "head"):
        dims = (1, cap, hkv, dh) if layout == "slot" else (1, hkv, cap, dh)
        exps = (1, cap // block, hkv) if layout == "slot" else (1, hkv, cap // block)
        d = {n: [torch.randint(0, 256, dims, generator=g, device="cuda", dtype=torch.uint8) & 0xB7] for n in "kv"}
        d.update({n + "_exp": [torch.randint(118, 122, exps, generator=g, device="cuda", dtype=torch.uint8)] for n in "kv"})
        n = cap - 200
        d.update(kv_block=block, seq_len=torch.tensor([n], dtype=torch.int32, device="cuda"),
                 tokens=torch.arange(cap, dtype=torch.int32, device="cuda")[None].contiguous(),
                 pos=torch.zeros(1, cap, dtype=torch.int32, device="cuda"), h2o_acc=torch.zeros(1, cap, device="cuda"))
        if layout == "head":
            d["kv_layout"] = cc.KV_HEAD_MAJOR
        cache = pkg.Cache(d)

        def last(name, m):   # the last slots of the sequence, as logical values
            x, e = d[name][0], d[name + "_exp"][0]
            if layout == "head":
                x, e = x.transpose(1, 2), e.transpose(1, 2)
            j = torch.arange(n + 100 - m, n + 100, device="cuda")
            return oracle.e4m3_decode(x[0, j].cpu().numpy()) * 2.0 ** (e[0, j // block].cpu().numpy().astype(int) - 127.0)[..., None]

        for m in (1, 100):
            q = torch.randn(m, hkv, dh, generator=g, device="cuda").to(torch.bfloat16)
            lse = torch.full((m, hkv), 14.0, device="cuda")
            rows = pkg.Rows(m, torch.tensor([0, m], dtype=torch.int32, device="cuda"), None, m)
            d["h2o_acc"].zero_()
            cc.cc_kv_accumulate(s, cache, 0, rows, q, lse, cc.alloc_workspace(cc.cc_kv_accumulate_workspace_size(s, cache, rows)))
            assert cc.cc_get_status() == cc.CC_OK
            k = last("k", tail)
            first = n + 100 - tail
            want, slack = oracle.received(q.double().cpu().numpy(), k[None], lse.cpu().numpy(), [n - first], [0, m])
            got = d["h2o_acc"][0, first:first + tail].cpu().numpy()
            assert (np.abs(got - want[0]) <= 2.0 ** -19 * slack[0] + 2.0 ** -14 * want[0]).all()
            assert (d["h2o_acc"][0, n + m:] == 0).all() and (d["h2o_acc"][0, :n + m] > 0).all()
        keep = np.unique(np.concatenate([np.arange(5), np.arange(n - 400, n, 3)]))
        idx = torch.zeros(1, cap, dtype=torch.int32, device="cuda")
        idx[0, :len(keep)] = torch.from_numpy(keep.astype(np.int32)).cuda()
        at = torch.from_numpy(keep).cuda()
        old = {}
        for name in "kv":
            x, e = d[name][0], d[name + "_exp"][0]
            if layout == "head":
                x, e = x.transpose(1, 2), e.transpose(1, 2)
            old[name] = (x[:, at].cpu().numpy(), e[:, at // block].cpu().numpy())
        cc.cc_kv_compact(s, cache, idx, torch.tensor([len(keep)], dtype=torch.int32, device="cuda"),
                         cc.alloc_workspace(cc.cc_kv_compact_workspace_size(s, cache)))
        assert cc.cc_get_status() == cc.CC_OK
        for name in "kv":
            x, e = d[name][0], d[name + "_exp"][0]
            if layout == "head":
                x, e = x.transpose(1, 2), e.transpose(1, 2)
            codes, each = old[name]
            tops = np.stack([each[0, j:j + block].max(0) for j in range(0, len(keep), block)])
            want = oracle.e4m3_encode(oracle.e4m3_decode(codes[0]) * 2.0 ** (each[0].astype(int) - np.repeat(tops, block, 0)[:len(keep)])[..., None])
            np.testing.assert_array_equal(x[0, :len(keep)].cpu().numpy(), want)
            np.testing.assert_array_equal(e[0, :len(tops)].cpu().numpy(), tops)
        np.testing.assert_array_equal(d["tokens"][0, :len(keep)].cpu().numpy(), keep)
        del d, cache


def test_a_dead_row_among_many_heads_behind_a_long_memory(pkg):
    """Slots so far before the rows that distance times heads passes 32 bits, next to a row that adds
    nothing (so that each weight is chosen).  Scores are 0: a slot gets the live rows' heads times e^-3.
    672 equal terms in fp32 differ from that by at most 672 * 2^-24, and each by under 2^-20."""
    from paper_2607_27600_gb300 import cc
    heads, dh, block, cap, m = 96, 64, 128, 1 << 25, 8
    n = cap - 256
    assert n * heads > 2 ** 31
    s = shape(heads, 1, dh)
    d = {x: [torch.zeros(1, cap, 1, dh, dtype=torch.uint8, device="cuda")] for x in "kv"}
    d.update({x + "_exp": [torch.full((1, cap // block, 1), 127, dtype=torch.uint8, device="cuda")] for x in "kv"})
    d.update(kv_block=block, seq_len=torch.tensor([n], dtype=torch.int32, device="cuda"),
             tokens=torch.zeros(1, cap, dtype=torch.int32, device="cuda"),
             pos=torch.zeros(1, cap, dtype=torch.int32, device="cuda"), h2o_acc=torch.zeros(1, cap, device="cuda"))
    cache = pkg.Cache(d)
    rows = pkg.Rows(m, torch.tensor([0, m], dtype=torch.int32, device="cuda"), None, m)
    q = torch.zeros(m, heads, dh, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((m, heads), 3.0, device="cuda")
    lse[3] = -float("inf")
    cc.cc_kv_accumulate(s, cache, 0, rows, q, lse, cc.alloc_workspace(cc.cc_kv_accumulate_workspace_size(s, cache, rows)))
    assert cc.cc_get_status() == cc.CC_OK
    live = torch.full((cap,), 7.0, dtype=torch.float64, device="cuda")
    live[n:n + m] = torch.tensor([7.0, 6, 5, 4, 4, 3, 2, 1], dtype=torch.float64, device="cuda")
    live[n + m:] = 0
    want = live * heads * math.exp(-3)
    assert ((d["h2o_acc"][0].double() - want).abs() <= (672 * 2.0 ** -24 + 2.0 ** -20) * want).all()
