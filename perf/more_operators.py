"""Performance cases of the operators by which a serving step's cache is managed:
what its slots receive, which of them stay, and attention over parts of a memory.

  received  cc_kv_accumulate: adds to the cache's running totals the attention that
            each slot receives from the new rows' queries, given the rows' log-sum-exp
  compact   cc_kv_compact: the kept slots of every layer of a block-format cache moved
            down in place, the codes of a new block brought to one scale, with the
            tokens, positions and totals
  join      cc_kv_join: attention over disjoint slots (a prefix that a batch shares and
            each sequence's own memory) joined by the parts' log-sum-exp

Shapes are the repository's: its tiny test shape, the Llama-3-8B and the
Qwen2.5-7B layer shapes.  With `own` false the operators are computed by
elementary torch operations in fp32; with `own` true by the library.
"""
import math

import torch

own = False

PAGE = 256   # slots per page of a paged cache
# layers, query heads, KV heads, head dim
MODELS = {"tiny": (1, 8, 2, 64), "llama8b": (32, 32, 8, 128), "qwen7b": (28, 28, 4, 128)}
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
NOT_NUMBERS = 255   # the scale exponent of a block whose elements are no numbers


def ints(text):
    return [int(x) for x in text.split(",")]


def cap_of(case):
    """Slots of the cache buffers, in whole pages."""
    grow = 0 if case.get("memory") or case["kind"] == "compact" else 1
    rows = ints(case["rows"]) if grow else [0] * len(ints(case["lens"]))
    return max(PAGE, -(-max(n + m for n, m in zip(ints(case["lens"]), rows)) // PAGE) * PAGE)


def spread(top, batch, least):
    """Lengths of a batch of sequences at different points of their cycles."""
    return ",".join(str(top - (top - least) * b // max(1, batch - 1)) for b in range(batch))


def each(value, batch):
    return ",".join([str(value)] * batch)


def shares(lens, part):
    """Slots that a refresh keeps of each length, at least one."""
    return ",".join(str(max(1, int(n * part))) if n else "0" for n in ints(lens))


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def received(name, model, lens, rows, dtype, layout, block, first=False, memory=False):
    return {"name": name, "kind": "received", "model": model, "lens": lens, "rows": rows, "dtype": dtype,
            "layout": layout, "block": block, "first": first, "memory": memory}


def compact(name, model, layers, lens, keep, layout, block):
    return {"name": name, "kind": "compact", "model": model, "layers": layers, "lens": lens, "keep": keep,
            "layout": layout, "block": block}


def join(name, model, rows, parts, dtype, pad=0):
    return {"name": name, "kind": "join", "model": model, "rows": rows, "parts": parts, "dtype": dtype, "pad": pad}


def listed():
    return [
        # one sequence's next token over the memory that a refresh kept: latency
        received("received-qwen-1", "qwen7b", "8191", "1", "bf16", "slot", 32),
        # a serving batch's next tokens, sequences of very different lengths: the keys read once
        received("received-llama-64", "llama8b", spread(32767, 64, 1500), each(1, 64), "bf16", "paged", 64,
                 first=True),
        # a few drafted tokens a sequence, checked together
        received("received-llama-draft", "llama8b", spread(9001, 16, 250), each(5, 16), "f16", "head", 128),
        # ragged chunks against the memory alone, one of them empty
        received("received-qwen-memory", "qwen7b", "8191,0,2049", "300,17,129", "f16", "slot", 16, memory=True),
        # a pre-fill chunk of one long sequence
        received("received-llama-chunk", "llama8b", "14336", "2048", "bf16", "paged", 64, first=True),
        # the smallest refresh: the repository's tiny workload
        compact("compact-tiny", "tiny", 1, "512", "128", "slot", 16),
        # every layer of a 16k memory down to a quarter
        compact("compact-llama-16k", "llama8b", 32, "16384", "4096", "paged", 64),
        # a ragged batch from which little is evicted, an empty sequence among them
        compact("compact-llama-batch", "llama8b", 4, "8192,0,5001,7777,130,16383",
                shares("8192,0,5001,7777,130,16383", 0.9), "slot", 32),
        # a long memory down to its budget, a head's slots together
        compact("compact-qwen-128k", "qwen7b", 4, "131072", "8192", "head", 128),
        # one decode step's row joined: latency
        join("join-qwen-1", "qwen7b", 1, 2, "bf16"),
        # a serving batch over a shared prefix, a document of its own and the recent tokens
        join("join-llama-300", "llama8b", 300, 3, "f16", 64),
        # chunks of a batch over a shared prefix and their own memory
        join("join-llama-8192", "llama8b", 8192, 2, "bf16"),
    ]


def between(rng, lo, hi):
    """A whole number, even over its logarithm; odd sizes as likely as even ones."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def fits(case):
    """A drawn case costs no more than the largest listed one of its kind, and
    the padded arrays of the plain form stay as small."""
    w = work(case)
    if case["kind"] == "join":
        return w["bytes"] <= 8192 * 32 * (3 * 256 + 12)
    lens = ints(case["lens"])
    layers, hq, hkv, dh = MODELS[case["model"]]
    held = len(lens) * cap_of(case) * hkv * dh
    if case["kind"] == "compact":
        moved = len(lens) * max(ints(case["keep"])) * hkv * dh * case["layers"]
        return (sum(ints(case["keep"])) > 0 and held * case["layers"] <= 32 * 16384 * 1024
                and w["bytes"] <= 5.4e8 and moved <= 2 * 32 * 4096 * 1024)
    rows = ints(case["rows"])
    scores = len(lens) * max(rows) * hq * max(n + m for n, m in zip(lens, rows))
    return (held <= 64 * 32768 * 1024 and scores <= 2048 * 16384 * 32 and w["flops"] <= 2.6e11
            and w["bytes"] <= 1.2e9 and sum(rows) > 0)


def draw(rng):
    while True:
        kind = rng.choice(["received", "received", "received", "compact", "compact", "join"])
        model = rng.choice(["tiny", "llama8b", "llama8b", "qwen7b", "qwen7b"])
        layout, block = rng.choice(["slot", "paged", "paged", "head"]), rng.choice([16, 32, 64, 128])
        if kind == "join":
            case = join("", model, between(rng, 1, 8192), rng.choice([2, 2, 3, 4, 8]),
                        rng.choice(["bf16", "bf16", "f16", "f32"]), rng.choice([0, 0, 8, 64]))
        elif kind == "compact":
            batch, top = between(rng, 1, 16), between(rng, 16, 131072)
            lens = [top] + [rng.choice([top, between(rng, 1, top), 0]) for _ in range(batch - 1)]
            lens = ",".join(map(str, lens))
            layers = 1 if model == "tiny" else between(rng, 1, MODELS[model][0])
            case = compact("", model, layers, lens, shares(lens, rng.choice([0.1, 0.25, 0.5, 0.75, 0.95])), layout, block)
        else:
            batch, most = between(rng, 1, 64), between(rng, 1, 2048)
            rows = [most] + [rng.choice([most, between(rng, 1, most), 0]) for _ in range(batch - 1)]
            top = between(rng, 16, 32768)
            lens = [rng.choice([top, between(rng, 1, top), between(rng, 1, top), 0]) for _ in range(batch)]
            memory = rng.random() < 0.25
            case = received("", model, ",".join(map(str, lens)), ",".join(map(str, rows)),
                            rng.choice(["bf16", "bf16", "f16"]), layout, block, not memory and rng.random() < 0.5,
                            memory)
        del case["name"]
        if fits(case):
            return case


def work(case):
    _, hq, hkv, dh = MODELS[case["model"]]
    if case["kind"] == "join":
        size, n, k = {"bf16": 2, "f16": 2, "f32": 4}[case["dtype"]], case["rows"] * hq, case["parts"]
        return {"bytes": n * (k + 1) * (dh * size + 4), "flops": 2 * n * k * dh}
    lens = ints(case["lens"])
    if case["kind"] == "compact":
        kept = sum(ints(case["keep"]))
        layer = 2 * kept * hkv * dh + 2 * kept * hkv // case["block"]
        return {"bytes": 2 * case["layers"] * layer + kept * (4 + 3 * 8), "flops": 0}
    rows, mem = ints(case["rows"]), case["memory"]
    seen = sum(a + (0 if mem else m) for a, m in zip(lens, rows) if m)
    pairs = sum(a * m + (0 if mem else m * (m + 1) // 2) for a, m in zip(lens, rows))
    return {"bytes": seen * hkv * dh + seen * hkv // case["block"] + seen * 8 + sum(rows) * hq * (2 * dh + 4),
            "flops": 2 * pairs * hq * dh}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

class State:
    pass


def places(st, b, slot):
    """Of slot `slot` of sequence `b` (index tensors of one shape): the index
    of each KV head's vector among a layer's vectors, and of its scale."""
    heads = torch.arange(st.hkv, device="cuda")
    b, slot = b.long()[..., None], slot.long()[..., None]
    if st.layout == "head":
        at = (b * st.hkv + heads) * st.cap + slot
        return at, at // st.block
    row = b * st.cap + slot
    if st.layout == "paged":
        row = st.table.long()[b, slot // PAGE] * PAGE + slot % PAGE
    return row * st.hkv + heads, row // st.block * st.hkv + heads


def power(e):
    """2^(e - 127) as fp32, e = 1 .. 254."""
    return (e.to(torch.int32) << 23).view(torch.float32)


def draw_cache(st, layers, held, g):
    """Codes and exponents of `layers` layers in the case's layout: N(0, s^2) with
    an s of each head's own, quantised block by block to the least scale that holds
    it; slots past a sequence's end (held[b] slots) hold any bits."""
    b = len(held)
    pages = b * st.cap // PAGE
    dims = {"slot": (b, st.cap, st.hkv, st.dh), "paged": (pages, PAGE, st.hkv, st.dh),
            "head": (b, st.hkv, st.cap, st.dh)}[st.layout]
    edims = {"slot": (b, st.cap // st.block, st.hkv), "paged": (pages, PAGE // st.block, st.hkv),
             "head": (b, st.hkv, st.cap // st.block)}[st.layout]
    codes = torch.randint(0, 256, (layers, *dims), generator=g, device="cuda", dtype=torch.uint8)
    exps = torch.randint(100, 150, (layers, *edims), generator=g, device="cuda", dtype=torch.uint8)
    std = torch.rand((layers, 1, st.hkv, 1), generator=g, device="cuda") * 1.5 + 0.5
    for layer in range(layers):
        for i, n in enumerate(held):
            if n == 0:
                continue
            full = -(-n // st.block) * st.block
            x = torch.randn((full // st.block, st.block, st.hkv, st.dh), generator=g, device="cuda") * std[layer]
            # now and then a block of larger values
            x *= 1 + 7 * (torch.rand((full // st.block, 1, st.hkv, 1), generator=g, device="cuda") < 0.1)
            mantissa, e = torch.frexp(x.abs().amax((1, 3)) / 448)
            e = e + 127 - (mantissa == 0.5).to(e.dtype)
            slot = torch.arange(n, device="cuda")
            at, eat = places(st, torch.full_like(slot, i), slot)
            y = (x * power(254 - e)[:, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
            codes[layer].view(-1, st.dh)[at.view(-1)] = y.reshape(full, st.hkv, st.dh)[:n].reshape(-1, st.dh)
            exps[layer].view(-1)[eat[:: st.block].reshape(-1)] = e.to(torch.uint8).view(-1)
    return codes, exps


def prepare(case, seed):
    """What a serving program holds before the call: the step's rows, the cache,
    the keep-set, buffers for the results, and the library's handles."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 71)
    st = State()
    st.kind = case["kind"]
    _, st.hq, st.hkv, st.dh = MODELS[case["model"]]
    if st.kind == "join":
        return prepare_join(st, case, g)
    st.lens, st.layout, st.block, st.cap = ints(case["lens"]), case["layout"], case["block"], cap_of(case)
    b = len(st.lens)
    st.table = None
    if st.layout == "paged":
        st.table = torch.randperm(b * st.cap // PAGE, generator=g, device="cuda").to(torch.int32)
        st.table = st.table.view(b, -1).contiguous()
    st.seq_len = torch.tensor(st.lens, dtype=torch.int32, device="cuda")
    st.tokens = torch.randint(0, 4096, (b, st.cap), generator=g, device="cuda", dtype=torch.int32)
    st.pos = torch.cumsum(torch.randint(1, 3, (b, st.cap), generator=g, device="cuda"), 1).to(torch.int32)
    # running totals of earlier steps: a few slots receive most of the attention
    st.acc = torch.rand((b, st.cap), generator=g, device="cuda").pow_(8).mul_(9)
    if st.kind == "compact":
        prepare_compact(st, case, g)
    else:
        prepare_received(st, case, g)
    if own:
        handles(st)
    return st


def prepare_received(st, case, g):
    st.dtype, st.rows = TYPES[case["dtype"]], ints(case["rows"])
    st.first, st.memory = case["first"], case["memory"]
    grown = [n + (0 if st.memory else m) for n, m in zip(st.lens, st.rows)]
    st.k_codes, st.k_exp = draw_cache(st, 1, grown, g)
    st.v_codes, st.v_exp = st.k_codes, st.k_exp   # (values take no part)
    st.n, st.max_rows = sum(st.rows), max(st.rows)
    st.acc *= 4 * st.hq * st.max_rows / st.cap   # (of about four steps like this one)
    starts = [0]
    for m in st.rows:
        starts.append(starts[-1] + m)
    st.row_start = torch.tensor(starts, dtype=torch.int32, device="cuda")
    # the queries, rotated, lie in the rows of a wider buffer
    wide = torch.randn((st.n, (st.hq + 2 * st.hkv) * st.dh), generator=g, device="cuda").mul_(1.25).to(st.dtype)
    st.q = wide[:, :st.hq * st.dh].view(st.n, st.hq, st.dh)
    # the log-sum-exp of the rows, as the step's attention leaves it
    s, seen = scores(st)
    lse = torch.logsumexp(s.masked_fill_(~seen, -math.inf), -1)
    seq, off = rows_of(st)
    st.lse = lse.permute(0, 2, 1, 3).reshape(len(st.lens), st.max_rows, st.hq)[seq, off].contiguous()


def prepare_compact(st, case, g):
    st.k_codes, st.k_exp = draw_cache(st, case["layers"], st.lens, g)
    st.v_codes, st.v_exp = draw_cache(st, case["layers"], st.lens, g)
    st.keep = ints(case["keep"])
    st.lens_before = st.seq_len.clone()
    st.keep_count = torch.tensor(st.keep, dtype=torch.int32, device="cuda")
    # the slots of the highest scores, the newest among them, in time order; what lies
    # behind them is not written
    st.keep_idx = torch.randint(-9, 1 << 20, (len(st.lens), st.cap), generator=g, device="cuda", dtype=torch.int32)
    for i, (n, k) in enumerate(zip(st.lens, st.keep)):
        if n:
            score = torch.rand(n, generator=g, device="cuda")
            score[-1] = 2
            st.keep_idx[i, :k] = score.topk(k).indices.sort().values.to(torch.int32)


def prepare_join(st, case, g):
    st.dtype, st.n = TYPES[case["dtype"]], case["rows"]
    width = st.hq * st.dh
    shape = (case["parts"], st.n, width + case["pad"])
    wide = torch.randn(shape, generator=g, device="cuda").to(st.dtype)
    st.parts = [x[:, :width].view(st.n, st.hq, st.dh) for x in wide]
    lse = torch.randn((case["parts"], st.n, st.hq), generator=g, device="cuda") * 1.5 + 8
    # a sequence whose own memory is empty: one row in 16 has nothing in the last part
    none = torch.arange(st.n, device="cuda") % 16 == 3
    lse[-1, none] = -math.inf
    st.parts[-1][none] = 0
    st.lses = list(lse)
    st.out = torch.empty((st.n, st.hq, st.dh), device="cuda", dtype=st.dtype)
    st.lse = torch.empty((st.n, st.hq), device="cuda")
    if own:
        from paper_2607_27600_gb300 import cc
        st.cfg = cc.cc_model_cfg(1, width, st.hq, st.hkv, st.dh, 4 * width, 4096, 1e4, 1e-5)
    return st


def handles(st):
    """The library's view of the cache and the rows, and its workspace."""
    import paper_2607_27600_gb300 as pkg
    from paper_2607_27600_gb300 import cc
    layers = st.k_codes.shape[0]
    st.cfg = cc.cc_model_cfg(layers, st.hq * st.dh, st.hq, st.hkv, st.dh, 4 * st.hq * st.dh, 4096, 1e4, 1e-5)
    d = {"k": list(st.k_codes), "v": list(st.v_codes), "k_exp": list(st.k_exp), "v_exp": list(st.v_exp),
         "kv_block": st.block, "seq_len": st.seq_len, "tokens": st.tokens, "pos": st.pos, "h2o_acc": st.acc}
    if st.layout == "paged":
        d["block_table"], d["page_size"] = st.table, PAGE
    if st.layout == "head":
        d["kv_layout"] = cc.KV_HEAD_MAJOR
    st.cache = pkg.Cache(d)
    if st.kind == "compact":
        st.ws = cc.alloc_workspace(cc.cc_kv_compact_workspace_size(st.cfg, st.cache))
    else:
        st.batch = pkg.Rows(st.n, row_start=st.row_start, max_rows=st.max_rows)
        st.ws = cc.alloc_workspace(cc.cc_kv_accumulate_workspace_size(st.cfg, st.cache, st.batch))


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(st):
    if st.kind == "compact":
        # the lengths as they were before the refresh, so that it can be run again
        st.seq_len.copy_(st.lens_before)
    if own:
        return run_own(st)
    return {"received": plain_received, "compact": plain_compact, "join": plain_join}[st.kind](st)


def run_own(st):
    from paper_2607_27600_gb300 import cc
    if st.kind == "received":
        cc.cc_kv_accumulate(st.cfg, st.cache, 0, st.batch, st.q, st.lse, st.ws, first=st.first,
                            memory_only=st.memory)
        return st.acc
    if st.kind == "compact":
        cc.cc_kv_compact(st.cfg, st.cache, st.keep_idx, st.keep_count, st.ws)
        return compacted(st)
    cc.cc_kv_join(st.cfg, st.parts, st.lses, st.out, lse=st.lse)
    return [st.out, st.lse]


def compacted(st):
    """The cache after the refresh: the codes as the e4m3 values they are, the scales'
    exponents, and what else a slot carries."""
    return [st.k_codes.view(torch.float8_e4m3fn), st.v_codes.view(torch.float8_e4m3fn), st.k_exp, st.v_exp,
            st.tokens, st.pos, st.acc, st.seq_len]


def rows_of(st):
    """Sequence and offset in it of every new row."""
    seq = torch.searchsorted(st.row_start[1:], torch.arange(st.n, device="cuda", dtype=torch.int32), right=True)
    return seq, torch.arange(st.n, device="cuda") - st.row_start[seq]


def scores(st):
    """q . k / sqrt(dh) as [batch, KV heads, rows, heads of a KV head, slots], and which
    of them a row sees (broadcast)."""
    b, g = len(st.lens), st.hq // st.hkv
    seq, off = rows_of(st)
    n_keys = max(1, max(st.lens) + (0 if st.memory else st.max_rows))
    n_keys = min(n_keys, st.cap)
    slot = torch.arange(n_keys, device="cuda")
    at, eat = places(st, torch.arange(b, device="cuda")[:, None].expand(b, n_keys), slot.expand(b, n_keys))
    count = st.row_start[1:] - st.row_start[:-1]
    held = slot < (st.seq_len if st.memory else st.seq_len + count)[:, None]
    k = st.k_codes.view(-1, st.dh)[at].view(torch.float8_e4m3fn).float()
    k *= power(st.k_exp.view(-1)[eat])[..., None]
    k.masked_fill_(~held[:, :, None, None], 0.0)                 # any bits past the end
    q = torch.zeros((b, st.max_rows, st.hq, st.dh), device="cuda")
    q[seq, off] = st.q.float()
    q = q.view(b, st.max_rows, st.hkv, g, st.dh).permute(0, 2, 1, 3, 4).reshape(b, st.hkv, -1, st.dh)
    s = torch.matmul(q, k.permute(0, 2, 3, 1))
    s *= 1 / math.sqrt(st.dh)
    row = torch.arange(st.max_rows, device="cuda")
    end = (st.seq_len[:, None] + (0 if st.memory else 1 + row)).expand(b, st.max_rows)
    end = torch.where(row < count[:, None], end, torch.zeros_like(end))   # rows of no one see nothing
    seen = (slot < end[..., None])[:, None, :, None]
    return s.view(b, st.hkv, st.max_rows, g, n_keys), seen


def plain_received(st):
    b = len(st.lens)
    seq, off = rows_of(st)
    s, seen = scores(st)
    lse = torch.full((b, st.max_rows, st.hq), math.inf, device="cuda")
    lse[seq, off] = torch.where(st.lse.isfinite(), st.lse, math.inf)   # a row without one adds nothing
    lse = lse.view(b, st.max_rows, st.hkv, -1).permute(0, 2, 1, 3)
    w = s.sub_(lse[..., None]).exp_().masked_fill_(~(seen & lse[..., None].isfinite()), 0.0)
    slot = torch.arange(st.cap, device="cuda")
    count = (st.row_start[1:] - st.row_start[:-1])[:, None]
    old = st.seq_len[:, None]
    if st.first:   # the new rows' slots begin at 0
        st.acc.masked_fill_((slot >= old) & (slot < old + count), 0.0)
    n_keys = w.shape[-1]
    st.acc[:, :n_keys] += w.sum((1, 2, 3))
    return st.acc


def plain_compact(st):
    b, most, blk = len(st.lens), max(st.keep), st.block
    planes = torch.arange(st.k_codes.shape[0], device="cuda")
    to = torch.arange(-(-most // blk) * blk, device="cuda")
    kept = to < st.keep_count[:, None]                                   # [b, slots]
    src = torch.where(kept, st.keep_idx[:, :to.numel()], 0).long()
    seq = torch.arange(b, device="cuda")[:, None].expand_as(kept)
    at, eat = places(st, seq, src)
    to_at, to_eat = places(st, seq, to.expand_as(kept))
    live = kept[:, :, None].expand_as(at)
    first = kept[:, ::blk, None].expand_as(to_eat[:, ::blk])             # blocks that hold a kept slot

    def move(codes, exps):
        layers = codes.shape[0]
        flat, eflat = codes.view(layers, -1, st.dh), exps.view(layers, -1)
        e = eflat[:, eat].to(torch.int32)                                # [layers, b, slots, hkv]
        bad = e == NOT_NUMBERS
        top = torch.where(live & ~bad, e, -1).view(layers, b, -1, blk, st.hkv).amax(3)
        top = torch.where(top < 0, NOT_NUMBERS, top)                     # (no number among them)
        new = top.repeat_interleave(blk, 2)
        x = flat[:, at].view(torch.float8_e4m3fn).float()
        scale = torch.where(e == 0, 0.0, power((127 + e - new).clamp(1, 254)))
        scale = torch.where(new == e, 1.0, scale)
        y = (x * scale[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
        y = torch.where((bad & (new != NOT_NUMBERS))[..., None], 0x7F, y)
        flat[:, to_at[live]] = y[:, live]
        eflat[:, to_eat[:, ::blk][first]] = top[:, first].to(torch.uint8)

    move(st.k_codes, st.k_exp)
    move(st.v_codes, st.v_exp)
    for x in (st.tokens, st.pos, st.acc):
        x[:, :to.numel()] = torch.where(kept, x.gather(1, src), x[:, :to.numel()])
    st.seq_len.copy_(st.keep_count)
    return compacted(st)


def plain_join(st):
    lse = torch.stack(st.lses)
    bad = (lse.isnan() | (lse == math.inf)).any(0)
    m = lse.amax(0)
    m = torch.where(m.isfinite(), m, torch.zeros_like(m))
    w = (lse - m).exp()
    total = w.sum(0)
    x = torch.stack(st.parts).float()
    x = torch.where(w[..., None] > 0, x, 0.0)   # a part without slots is not looked at
    y = (x * w[..., None]).sum(0) / torch.where(total > 0, total, 1.0)[..., None]
    y = torch.where(bad[..., None], 0.0, y)
    return [y.to(st.dtype), torch.where(bad, math.nan, m + total.log())]


# ---------------------------------------------------------------------------
# from the definitions, in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    return {"received": exact_received, "compact": exact_compact, "join": exact_join}[st.kind](st)


def value_table():
    """The 256 e4m3 codes' values, from the format's fields."""
    c = torch.arange(256, device="cuda")
    e, m = (c >> 3) & 15, (c & 7).double() / 8
    x = torch.where(e > 0, (1 + m) * torch.exp2((e - 7).double()), m * 2.0 ** -6)
    x = torch.where((c & 127) == 127, math.nan, x)
    return torch.where(c < 128, x, -x)


def exact_received(st):
    table, g = value_table(), st.hq // st.hkv
    acc = st.acc.double()
    lo = 0
    for i, (n, m) in enumerate(zip(st.lens, st.rows)):
        end = n if st.memory else n + m
        if st.first:
            acc[i, n:n + m] = 0
        if m and end:
            slot = torch.arange(end, device="cuda")
            at, eat = places(st, torch.full_like(slot, i), slot)
            sees = torch.full((m,), n, device="cuda") if st.memory else n + 1 + torch.arange(m, device="cuda")
            for h in range(st.hq):
                k = table[st.k_codes.view(-1, st.dh)[at[:, h // g]].int()]
                k = k * torch.exp2(st.k_exp.view(-1)[eat[:, h // g]].double() - 127)[:, None]
                s = st.q[lo:lo + m, h].double() @ k.T / math.sqrt(st.dh) - st.lse[lo:lo + m, h].double()[:, None]
                acc[i, :end] += torch.where(slot < sees[:, None], s.exp(), 0.0).sum(0)
        lo += m
    return acc


def nearest_code_value(x):
    """The nearest e4m3 value, ties to the even code, of |x| <= 448."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -40))).clamp(min=-6)
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def exact_compact(st):
    table, outs, new_exps = value_table(), [], []
    for codes, exps in ((st.k_codes, st.k_exp), (st.v_codes, st.v_exp)):
        values, exps = [], exps.clone()
        for layer in range(codes.shape[0]):
            before = codes[layer].view(-1, st.dh)
            out = table[before.int()].view(codes.shape[1:])
            flat, eflat = out.view(-1, st.dh), exps[layer].view(-1)
            for i, k in enumerate(st.keep):
                if k == 0:
                    continue
                src = st.keep_idx[i, :k].long()
                at, eat = places(st, torch.full_like(src, i), src)
                to = torch.arange(k, device="cuda")
                to_at, to_eat = places(st, torch.full_like(to, i), to)
                e = eflat[eat].double()                                  # [k, hkv]
                pad = torch.nn.functional.pad(e, (0, 0, 0, -k % st.block))
                top = pad.view(-1, st.block, st.hkv).amax(1)             # (inputs of a draw: 1 .. 254)
                x = table[before[at].int()] * torch.exp2(e - top.repeat_interleave(st.block, 0)[:k])[..., None]
                flat[to_at] = nearest_code_value(x)
                eflat[to_eat[:: st.block]] = top.to(torch.uint8)
            values.append(out)
        outs.append(torch.stack(values))
        new_exps.append(exps)
    rest = []
    for x in (st.tokens, st.pos, st.acc):
        y = x.clone()
        for i, k in enumerate(st.keep):
            y[i, :k] = x[i, st.keep_idx[i, :k].long()]
        rest.append(y.double() if y.is_floating_point() else y)
    return [*outs, *new_exps, *rest, torch.tensor(st.keep, dtype=torch.int32, device="cuda")]


def exact_join(st):
    lse = torch.stack(st.lses).double()
    p = torch.softmax(lse, 0)   # (a part of every row of a draw has slots)
    out = sum(w[..., None] * x.double() for w, x in zip(p, st.parts))
    return [out, torch.logsumexp(lse, 0)]
