"""Performance cases of the operators that a serving step is made of when the
model's own code computes the projections: the cache write, the attention that
reads it, and the answer.

  append    cc_kv_append: the new tokens' queries and keys rotated at their
            positions, keys and values written into the cache's slots as 8-bit
            codes with a power-of-two scale for each block of slots and KV head
  attend    cc_kv_attention: the new tokens' queries against that cache, with
            the log-sum-exp of each row
  logprob   cc_token_logprobs: each row's log-probability of a given token, its
            entropy and its most likely alternatives

Shapes are the repository's: its tiny test shape, the Llama-3-8B and the
Qwen2.5-7B layer shapes.  With `own` false the operators are computed by
elementary torch operations in fp32; with `own` true by the library.
"""
import math

import torch

own = False

PAGE = 256   # slots per page of a paged cache
# query heads, KV heads, head dim, vocabulary, RoPE base
MODELS = {
    "tiny": (8, 2, 64, 4096, 1e4),
    "llama8b": (32, 8, 128, 128256, 5e5),
    "qwen7b": (28, 4, 128, 152064, 1e6),
}
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
LEAST_EXP, MOST_EXP, UNIT_EXP = 10, 247, 127   # scale exponents that are written; scale 1, of zeros


def ints(text):
    return [int(x) for x in text.split(",")]


def cap_of(case):
    """Slots of the cache buffers, in whole pages."""
    grow = 0 if case.get("memory") else 1
    need = max(n + m * grow for n, m in zip(ints(case["lens"]), ints(case["rows"])))
    return max(PAGE, -(-need // PAGE) * PAGE)


def spread(top, batch, least):
    """Lengths of a batch of sequences at different points of their cycles."""
    return ",".join(str(top - (top - least) * b // max(1, batch - 1)) for b in range(batch))


def each(value, batch):
    return ",".join([str(value)] * batch)


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def append(name, model, lens, rows, dtype, layout, block):
    return {"name": name, "kind": "append", "model": model, "lens": lens, "rows": rows,
            "dtype": dtype, "layout": layout, "block": block}


def attend(name, model, lens, rows, dtype, layout, block, memory=False):
    return {"name": name, "kind": "attend", "model": model, "lens": lens, "rows": rows,
            "dtype": dtype, "layout": layout, "block": block, "memory": memory}


def logprob(name, model, rows, dtype, top, pad=0, masked=False):
    return {"name": name, "kind": "logprob", "model": model, "rows": rows, "dtype": dtype,
            "top": top, "pad": pad, "masked": masked}


def listed():
    return [
        # one sequence's next token over the memory that a refresh kept: latency
        append("append-qwen-1", "qwen7b", "8191", "1", "bf16", "slot", 32),
        # a serving batch's next tokens into a paged cache
        append("append-llama-64", "llama8b", spread(2000, 64, 33), each(1, 64), "bf16", "paged", 64),
        # ragged prompts of odd lengths, a single token and nothing at all among
        # them, from fp32 projections, into a cache that keeps a head's slots together
        append("append-qwen-ragged", "qwen7b", "100,0,4095,1000,7", "777,2049,1,0,130", "f32", "head",
               16),
        # four prompts of the chunked pre-fill
        append("append-llama-16k", "llama8b", "8192,4096,0,5", "4096,4096,4096,4096", "bf16", "paged",
               128),
        # one sequence's next token over the memory that a refresh kept
        attend("attend-qwen-1", "qwen7b", "8191", "1", "bf16", "slot", 32),
        # a serving batch of sequences of very different lengths, the cache read once
        attend("attend-llama-64", "llama8b", spread(32767, 64, 1500), each(1, 64), "bf16", "paged", 64),
        # a few drafted tokens a sequence, checked together
        attend("attend-llama-draft", "llama8b", spread(9001, 16, 250), each(5, 16), "f16", "head", 128),
        # queries over the memory alone (one of them empty), to be joined with
        # attention over tokens held elsewhere
        attend("attend-qwen-memory", "qwen7b", "8191,0,2049", "300,17,129", "bf16", "slot", 16, True),
        # a pre-fill chunk of one long sequence
        attend("attend-llama-chunk", "llama8b", "14336", "2048", "bf16", "paged", 64),
        # the answer of one decode step
        logprob("logprob-llama-1", "llama8b", 1, "f32", 20),
        # a serving batch whose sampler forbids tokens, rows padded to a wider pitch
        logprob("logprob-qwen-64", "qwen7b", 64, "bf16", 5, 64, True),
        # the log-probabilities of a whole prompt
        logprob("logprob-llama-4096", "llama8b", 4096, "bf16", 8),
    ]


def between(rng, lo, hi):
    """A whole number, even over its logarithm; odd sizes as likely as even ones."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def fits(case):
    """A drawn case costs no more than the largest listed one of its kind, and
    the padded arrays of the plain form stay as small."""
    w = work(case)
    if case["kind"] == "logprob":
        return w["bytes"] <= 4096 * 128256 * 2 * 1.01
    lens, rows = ints(case["lens"]), ints(case["rows"])
    hq, hkv, dh, _, _ = MODELS[case["model"]]
    if case["kind"] == "append":
        return sum(rows) <= 16384 and len(rows) * max(rows) <= 32768 and len(rows) * cap_of(case) <= 131072
    held = len(lens) * cap_of(case) * hkv * dh
    scores = len(lens) * max(rows) * hq * max(n + m for n, m in zip(lens, rows))
    return (held <= 64 * 32768 * 8 * 128 and scores <= 2048 * 16384 * 32 and w["flops"] <= 5e11
            and sum(rows) > 0)


def draw(rng):
    while True:
        kind = rng.choice(["append", "append", "attend", "attend", "attend", "logprob", "logprob"])
        model = rng.choice(["tiny", "llama8b", "llama8b", "qwen7b", "qwen7b"])
        if kind == "logprob":
            case = logprob("", model, between(rng, 1, 4096), rng.choice(["bf16", "bf16", "f16", "f32"]),
                           between(rng, 1, 32), rng.choice([0, 0, 8, 37]), rng.random() < 0.3)
        else:
            batch = between(rng, 1, 64)
            most = between(rng, 1, 4096 if kind == "append" else 2048)
            rows = [most] + [rng.choice([most, between(rng, 1, most), 0]) for _ in range(batch - 1)]
            top = between(rng, 16, 32768)
            lens = [rng.choice([top, between(rng, 1, top), between(rng, 1, top), 0]) for _ in range(batch)]
            common = (model, ",".join(map(str, lens)), ",".join(map(str, rows)))
            layout = rng.choice(["slot", "paged", "paged", "head"])
            block = rng.choice([16, 32, 64, 128])
            if kind == "append":
                case = append("", *common, rng.choice(["bf16", "bf16", "f16", "f32"]), layout, block)
            else:
                case = attend("", *common, rng.choice(["bf16", "bf16", "f16"]), layout, block,
                              rng.random() < 0.25)
        del case["name"]
        if fits(case):
            return case


def work(case):
    hq, hkv, dh, vocab, _ = MODELS[case["model"]]
    size = {"bf16": 2, "f16": 2, "f32": 4}[case["dtype"]]
    if case["kind"] == "logprob":
        r, k = case["rows"], case["top"]
        return {"bytes": r * vocab * size + r * (12 + 8 * k), "flops": 4 * r * vocab}
    lens, rows = ints(case["lens"]), ints(case["rows"])
    n = sum(rows)
    if case["kind"] == "append":
        codes = 2 * n * hkv * dh
        return {"bytes": n * (2 * hq + 2 * hkv) * dh * size + codes + codes // dh // case["block"],
                "flops": 3 * n * (hq + hkv) * dh}
    mem = case["memory"]
    seen = sum(a + (0 if mem else m) for a, m in zip(lens, rows) if m)
    pairs = sum(a * m + (0 if mem else m * (m + 1) // 2) for a, m in zip(lens, rows))
    return {"bytes": 2 * seen * hkv * dh + 2 * seen * hkv // case["block"] + n * hq * (2 * dh * size + 4),
            "flops": 4 * pairs * hq * dh}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

class State:
    pass


def places(st, b, slot):
    """Of slot `slot` of sequence `b` (index tensors of one shape): the index
    of each KV head's vector among the buffer's vectors, and of its scale."""
    heads = torch.arange(st.hkv, device="cuda")
    b, slot = b.long()[..., None], slot.long()[..., None]
    if st.layout == "head":
        at = (b * st.hkv + heads) * st.cap + slot
        return at, at // st.block
    row = b * st.cap + slot
    if st.layout == "paged":
        row = st.table.long()[b, slot // PAGE] * PAGE + slot % PAGE
    return row * st.hkv + heads, row // st.block * st.hkv + heads


def pair_bound(x):
    """An upper bound of the radius of every rotate-half pair of x (.., dh):
    max + min / 2 >= sqrt(a^2 + b^2), whatever the rotation."""
    a, b = x.abs().chunk(2, dim=-1)
    return torch.maximum(a, b) + 0.5 * torch.minimum(a, b)


def exponent(bound):
    """The least exponent e with bound <= 448 * 2^(e - 127), in the written
    range; 0 where the bound is 0 and any scale would do."""
    bits = bound.contiguous().view(torch.int32)
    e = ((bits + 0x1FFFFF) >> 23) - 8   # 448 = 1.75 * 2^8: past mantissa .75 the next power
    e = e.clamp(LEAST_EXP, MOST_EXP)
    return torch.where(bound > 0, e, torch.zeros_like(e))


def power(e):
    """2^(e - 127) as fp32."""
    return (e.to(torch.int32) << 23).view(torch.float32)


def codes_of(x, e):
    """x / 2^(e - 127) rounded to e4m3 codes; an infinity becomes NaN."""
    y = x * power(254 - e)[..., None]
    return torch.where(x.isinf(), torch.full_like(y, math.nan), y).to(torch.float8_e4m3fn)


def finite_abs(x):
    return torch.where(x.isfinite(), x, torch.zeros_like(x))


def draw_cache(st, case, g):
    """K and V in the case's layout: the memory (for attention after an append,
    the new tokens too), values N(0, s^2) with s of each head its own,
    quantised block by block; slots past a sequence's end hold any bits."""
    b = len(st.lens)
    dims = {"slot": (b, st.cap, st.hkv, st.dh), "paged": (b * st.cap // PAGE, PAGE, st.hkv, st.dh),
            "head": (b, st.hkv, st.cap, st.dh)}[st.layout]
    edims = {"slot": (b, st.cap // st.block, st.hkv), "paged": (b * st.cap // PAGE, PAGE // st.block, st.hkv),
             "head": (b, st.hkv, st.cap // st.block)}[st.layout]
    out = []
    for _ in range(2):
        codes = torch.randint(0, 256, dims, generator=g, device="cuda", dtype=torch.uint8)
        exps = torch.randint(100, 150, edims, generator=g, device="cuda", dtype=torch.uint8)
        std = torch.rand((st.hkv, 1), generator=g, device="cuda") * 1.5 + 0.5
        for i, (n, m) in enumerate(zip(st.lens, st.rows)):
            n += m if st.kind == "attend" and not st.memory else 0
            if n == 0:
                continue
            x = torch.randn((n, st.hkv, st.dh), generator=g, device="cuda") * std
            pad = -n % st.block
            full = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, pad)) if pad else x
            e = exponent(full.abs().view(-1, st.block, st.hkv, st.dh).amax((1, 3)))
            slot = torch.arange(n, device="cuda")
            at, eat = places(st, torch.full_like(slot, i), slot)
            codes.view(-1, st.dh)[at.view(-1)] = \
                codes_of(x, e.repeat_interleave(st.block, 0)[:n]).view(torch.uint8).view(-1, st.dh)
            exps.view(-1)[eat[:: st.block].reshape(-1)] = e.to(torch.uint8).view(-1)
        out += [codes, exps]
    return out


def prepare(case, seed):
    """What a serving program holds before the call: the projections' output
    rows, the cache, buffers for the results, and the library's handles."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 29)
    st = State()
    st.kind, st.dtype = case["kind"], TYPES[case["dtype"]]
    st.hq, st.hkv, st.dh, st.vocab, st.theta = MODELS[case["model"]]
    if st.kind == "logprob":
        n, st.top = case["rows"], case["top"]
        z = torch.randn((n, st.vocab + case["pad"]), generator=g, device="cuda", dtype=torch.float32)
        st.logits = z.mul_(2.5).to(st.dtype)[:, :st.vocab]   # the pitch may be wider than a row
        st.targets = torch.randint(0, st.vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
        if case["masked"]:   # one row in four allows one token in 64, the target among them
            for r in range(0, n, 4):
                st.logits[r].masked_fill_((torch.arange(st.vocab, device="cuda") - st.targets[r]) % 64 != 0,
                                          -math.inf)
        st.logprob = torch.empty(n, device="cuda")
        st.entropy = torch.empty(n, device="cuda")
        st.top_ids = torch.empty((n, st.top), device="cuda", dtype=torch.int32)
        st.top_logprob = torch.empty((n, st.top), device="cuda")
        return st
    st.lens, st.rows = ints(case["lens"]), ints(case["rows"])
    st.layout, st.block, st.cap = case["layout"], case["block"], cap_of(case)
    st.memory = case.get("memory", False)
    b, n = len(st.lens), sum(st.rows)
    st.table = None
    if st.layout == "paged":
        st.table = torch.randperm(b * st.cap // PAGE, generator=g, device="cuda").to(torch.int32)
        st.table = st.table.view(b, -1).contiguous()
    st.k_codes, st.k_exp, st.v_codes, st.v_exp = draw_cache(st, case, g)
    st.seq_len = torch.tensor(st.lens, dtype=torch.int32, device="cuda")
    starts = [0]
    for m in st.rows:
        starts.append(starts[-1] + m)
    st.n, st.max_rows = n, max(st.rows)
    st.row_start = torch.tensor(starts, dtype=torch.int32, device="cuda")
    # positions run ahead of the slots: the memory has lost evicted tokens
    ahead = torch.randint(0, 8192, (b,), generator=g, device="cuda")
    seq = torch.repeat_interleave(torch.arange(b, device="cuda"), torch.tensor(st.rows, device="cuda"))
    st.pos = (st.seq_len[seq] + torch.arange(n, device="cuda") - st.row_start[seq] + ahead[seq]).to(torch.int32)
    # q, k and v lie side by side in the rows of one projection
    width = (st.hq + 2 * st.hkv) * st.dh
    qkv = torch.randn((n, width), generator=g, device="cuda", dtype=torch.float32).mul_(1.25).to(st.dtype)
    st.q = qkv[:, :st.hq * st.dh].view(n, st.hq, st.dh)
    st.k = qkv[:, st.hq * st.dh:(st.hq + st.hkv) * st.dh].view(n, st.hkv, st.dh)
    st.v = qkv[:, (st.hq + st.hkv) * st.dh:].view(n, st.hkv, st.dh)
    st.out = torch.empty((n, st.hq, st.dh), device="cuda", dtype=st.dtype)
    st.lse = torch.empty((n, st.hq), device="cuda")
    st.turns = torch.tensor([turn - (1 << 64) if turn >= 1 << 63 else turn for turn in
                             (int(math.ldexp(st.theta ** (-2.0 * i / st.dh) / (2 * math.pi), 64))
                              for i in range(st.dh // 2))], dtype=torch.int64, device="cuda")
    if own:
        handles(st)
    return st


def handles(st):
    """The library's view of the cache and the rows, and its workspace."""
    import paper_2607_27600_gb300 as pkg
    from paper_2607_27600_gb300 import cc
    b = len(st.lens)
    st.cfg = cc.cc_model_cfg(1, st.hq * st.dh, st.hq, st.hkv, st.dh, 4 * st.hq * st.dh, st.vocab,
                             st.theta, 1e-5)
    d = {"k": [st.k_codes], "v": [st.v_codes], "k_exp": [st.k_exp], "v_exp": [st.v_exp],
         "kv_block": st.block, "seq_len": st.seq_len,
         "tokens": torch.zeros((b, st.cap), dtype=torch.int32, device="cuda"),
         "pos": torch.zeros((b, st.cap), dtype=torch.int32, device="cuda")}
    if st.layout == "paged":
        d["block_table"], d["page_size"] = st.table, PAGE
    if st.layout == "head":
        d["kv_layout"] = cc.KV_HEAD_MAJOR
    st.cache = pkg.Cache(d)
    st.batch = pkg.Rows(st.n, row_start=st.row_start, pos=st.pos, max_rows=st.max_rows)
    st.ws = cc.alloc_workspace(cc.cc_kv_attention_workspace_size(st.cfg, st.cache, st.batch))


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(st):
    if own:
        return run_own(st)
    return {"append": plain_append, "attend": plain_attend, "logprob": plain_logprob}[st.kind](st)


def run_own(st):
    from paper_2607_27600_gb300 import cc
    if st.kind == "append":
        cc.cc_kv_append(st.cfg, st.cache, 0, st.batch, st.k, st.v, st.q, st.out)
        return appended(st, st.out)
    if st.kind == "attend":
        cc.cc_kv_attention(st.cfg, st.cache, 0, st.batch, st.q, st.out, st.ws, lse=st.lse,
                           memory_only=st.memory)
        return [st.out, st.lse]
    cc.cc_token_logprobs(st.logits, st.targets, st.logprob, st.entropy, st.top_ids, st.top_logprob)
    return [st.logprob, st.entropy, st.top_ids, st.top_logprob]


def appended(st, q):
    """The rotated queries and the cache after the append: the codes as the
    e4m3 values they are, and the scales' exponents."""
    return [q, st.k_codes.view(torch.float8_e4m3fn), st.v_codes.view(torch.float8_e4m3fn), st.k_exp, st.v_exp]


def rotate(st, x):
    """Rotate-half pairs of x [n, heads, dh] at the rows' positions.  The
    angle is reduced exactly: pos * turns mod 2^64 is a fraction of a turn."""
    frac = st.pos.long()[:, None] * st.turns   # wraps modulo 2^64
    angle = (frac >> 32).to(torch.float32) * (2 * math.pi / 2 ** 32)
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    a, b = x.float().chunk(2, dim=-1)
    return torch.cat([a * c - b * s, b * c + a * s], dim=-1)


def rows_of(st):
    """Sequence and offset in it of every new row."""
    seq = torch.searchsorted(st.row_start[1:], torch.arange(st.n, device="cuda", dtype=torch.int32), right=True)
    return seq, torch.arange(st.n, device="cuda") - st.row_start[seq]


def plain_append(st):
    b, blk = len(st.lens), st.block
    seq, off = rows_of(st)
    first = st.seq_len // blk                      # first block that is written
    slot = st.seq_len[seq] + off
    q, k, v = rotate(st, st.q), rotate(st, st.k), st.v.float()
    nb = (st.max_rows + blk - 2) // blk + 1        # blocks that a sequence's rows touch at most
    j = slot // blk - first[seq]
    new = torch.zeros((b, nb, blk), dtype=torch.bool, device="cuda")
    new[seq, j, slot % blk] = True
    # the memory's slots of the first block
    held = (torch.arange(blk, device="cuda") < (st.seq_len % blk)[:, None]) & new[:, 0].any(1, keepdim=True)
    old_at, old_eat = places(st, torch.arange(b, device="cuda")[:, None].expand(b, blk),
                             (first[:, None] * blk + torch.arange(blk, device="cuda")).clamp(max=st.cap - 1))
    some = held[:, 0]                              # it holds older slots
    at, eat = places(st, seq, slot)

    def write(x, bound, codes, exps):
        flat, eflat = codes.view(-1, st.dh), exps.view(-1)
        top = torch.zeros((b, nb, blk, st.hkv), device="cuda")
        top[seq, j, slot % blk] = bound.amax(-1)
        e = exponent(top.amax(2))                                   # [b, nb, hkv]
        e_old = eflat[old_eat[:, 0]].to(torch.int32)                # [b, hkv]
        e[:, 0] = torch.where(some[:, None], torch.maximum(e[:, 0], e_old), e[:, 0])
        e = torch.where(e == 0, torch.full_like(e, UNIT_EXP), e)
        old = flat[old_at].view(torch.float8_e4m3fn).float()        # [b, blk, hkv, dh]
        scaled = (old * power((127 + e_old - e[:, 0]).clamp(min=1))[:, None, :, None]).to(torch.float8_e4m3fn)
        flat[old_at] = torch.where(held[:, :, None, None], scaled.view(torch.uint8), flat[old_at])
        flat[at] = codes_of(x, e[seq, j]).view(torch.uint8)
        eflat[eat] = e[seq, j].to(torch.uint8)

    write(k, pair_bound(finite_abs(st.k.float())), st.k_codes, st.k_exp)
    write(v, finite_abs(v).abs(), st.v_codes, st.v_exp)
    return appended(st, q.to(st.dtype))


def plain_attend(st):
    b, g = len(st.lens), st.hq // st.hkv
    seq, off = rows_of(st)
    n_keys = max(1, min(st.cap, max(st.lens) + (0 if st.memory else st.max_rows)))
    slot = torch.arange(n_keys, device="cuda")
    at, eat = places(st, torch.arange(b, device="cuda")[:, None].expand(b, n_keys), slot.expand(b, n_keys))
    count = st.row_start[1:] - st.row_start[:-1]
    n_seen = st.seq_len if st.memory else st.seq_len + count
    seen = slot < n_seen[:, None]                                    # [b, keys]

    def values(codes, exps):
        x = codes.view(-1, st.dh)[at].view(torch.float8_e4m3fn).float()
        x *= power(exps.view(-1)[eat])[..., None]
        x.masked_fill_(~seen[:, :, None, None], 0.0)                 # any bits past the end
        return x.transpose(1, 2)                                     # [b, hkv, keys, dh]

    q = torch.zeros((b, st.max_rows, st.hq, st.dh), device="cuda")
    q[seq, off] = st.q.float()
    q = q.view(b, st.max_rows, st.hkv, g, st.dh).permute(0, 2, 1, 3, 4).reshape(b, st.hkv, -1, st.dh)
    s = torch.matmul(q, values(st.k_codes, st.k_exp).transpose(-1, -2))
    s *= 1 / math.sqrt(st.dh)
    end = n_seen[:, None] if st.memory else st.seq_len[:, None] + 1 + torch.arange(st.max_rows, device="cuda")
    end = end.expand(b, st.max_rows)
    s = s.view(b, st.hkv, st.max_rows, g, n_keys)
    s.masked_fill_(~(slot < end[..., None])[:, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(b, st.hkv, -1, n_keys), values(st.v_codes, st.v_exp))
    o = o.view(b, st.hkv, st.max_rows, g, st.dh) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (m + total.log()).squeeze(-1)
    o = o.permute(0, 2, 1, 3, 4).reshape(b, st.max_rows, st.hq, st.dh)
    lse = lse.permute(0, 2, 1, 3).reshape(b, st.max_rows, st.hq)
    return [o[seq, off].to(st.dtype), lse[seq, off]]


def plain_logprob(st):
    z = st.logits.float()
    m = z.amax(-1, keepdim=True)
    d = z - m
    e = d.exp()
    total = e.sum(-1)
    log_total = total.log()
    lse = m[:, 0] + log_total
    entropy = log_total - torch.where(e > 0, e * d, torch.zeros_like(e)).sum(-1) / total
    lp = z.gather(1, st.targets.long()[:, None])[:, 0] - lse
    # the largest values, ties to the lowest id: one whole number orders both
    bits = (z + 0.0).view(torch.int32)
    bits = bits ^ ((bits >> 31) & 0x7FFFFFFF)
    keys = (bits.long() << 32) | (st.vocab - 1 - torch.arange(st.vocab, device="cuda"))
    ids = st.vocab - 1 - (keys.topk(st.top, dim=-1).values & 0xFFFFFFFF)
    return [lp, entropy, ids.to(torch.int32), z.gather(1, ids) - lse[:, None]]


# ---------------------------------------------------------------------------
# from the definitions, in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    return {"append": exact_append, "attend": exact_attend, "logprob": exact_logprob}[st.kind](st)


def exact_value(codes, exps):
    """e4m3 codes (uint8) with their blocks' exponents, from the format's fields."""
    c = codes.to(torch.int64)
    sign, e, m = 1 - 2 * (c >> 7).double(), (c >> 3) & 15, (c & 7).double()
    x = torch.where(e > 0, (1 + m / 8) * torch.exp2((e - 7).double()), m / 8 * 2.0 ** -6)
    x = torch.where((c & 127) == 127, torch.full_like(x, math.nan), x)
    return sign * x * torch.exp2(exps.double() - 127)


def exact_round(x):
    """The nearest e4m3 value, ties to even, at most 448 in magnitude."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -60))).clamp(min=-6)
    step = torch.exp2(e - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def exact_rotate(st, x):
    freq = st.theta ** (-2.0 * torch.arange(st.dh // 2, device="cuda", dtype=torch.float64) / st.dh)
    angle = (st.pos.double()[:, None] * freq)[:, None]
    a, b = x.double()[..., :st.dh // 2], x.double()[..., st.dh // 2:]
    return torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1)


def exact_append(st):
    outs = []
    half = st.dh // 2
    a, b = st.k.double()[..., :half].abs(), st.k.double()[..., half:].abs()
    k_top = (torch.maximum(a, b) + torch.minimum(a, b) / 2).float().double()   # (an fp32 sum)
    for x, top, codes, exps in ((exact_rotate(st, st.k), k_top.amax(-1), st.k_codes, st.k_exp),
                                (st.v.double(), st.v.double().abs().amax(-1), st.v_codes, st.v_exp)):
        values = codes.view(torch.float8_e4m3fn).double()
        exps = exps.clone()
        flat, eflat = values.view(-1, st.dh), exps.view(-1)
        lo = 0
        for i, (n, m) in enumerate(zip(st.lens, st.rows)):
            done = 0
            while done < m:
                s0 = n + done
                s1 = min(n + m, (s0 // st.block + 1) * st.block)
                r = slice(lo + done, lo + done + s1 - s0)
                slots = torch.arange(s0 // st.block * st.block, s1, device="cuda")
                at, eat = places(st, torch.full_like(slots, i), slots)
                held = s0 % st.block
                need = torch.ceil(torch.log2(top[r].amax(0) / 448)) + 127   # (inputs of a draw: never 0)
                need = need.clamp(LEAST_EXP, MOST_EXP)
                before = eflat[eat[0]].double()
                e = torch.maximum(need, before) if held else need
                if held:
                    flat[at[:held]] = exact_round(flat[at[:held]] * torch.exp2(before - e)[:, None])
                flat[at[held:]] = exact_round(x[r] / torch.exp2(e - 127)[:, None])
                eflat[eat[0]] = e.to(torch.uint8)
                done += s1 - s0
            lo += m
        outs.append((values, exps))
    (k, ke), (v, ve) = outs
    return [exact_rotate(st, st.q), k, v, ke, ve]


def exact_attend(st):
    out = torch.zeros((st.n, st.hq, st.dh), device="cuda", dtype=torch.float64)
    lse = torch.full((st.n, st.hq), -math.inf, device="cuda", dtype=torch.float64)
    lo, g = 0, st.hq // st.hkv
    for i, (n, m) in enumerate(zip(st.lens, st.rows)):
        end = n if st.memory else n + m
        if m and end:
            slot = torch.arange(end, device="cuda")
            at, eat = places(st, torch.full_like(slot, i), slot)
            for h in range(st.hkv):
                k = exact_value(st.k_codes.view(-1, st.dh)[at[:, h]], st.k_exp.view(-1)[eat[:, h]][:, None])
                v = exact_value(st.v_codes.view(-1, st.dh)[at[:, h]], st.v_exp.view(-1)[eat[:, h]][:, None])
                q = st.q[lo:lo + m, h * g:(h + 1) * g].double().reshape(m * g, st.dh)
                s = q @ k.T / math.sqrt(st.dh)
                if not st.memory:
                    row = n + torch.arange(m, device="cuda").repeat_interleave(g)
                    s = s.masked_fill(slot > row[:, None], -math.inf)
                out[lo:lo + m, h * g:(h + 1) * g] = (torch.softmax(s, -1) @ v).view(m, g, st.dh)
                lse[lo:lo + m, h * g:(h + 1) * g] = torch.logsumexp(s, -1).view(m, g)
        lo += m
    return [out, lse]


def exact_logprob(st):
    parts = [[], [], []]
    ids = []
    for r in range(0, st.logits.shape[0], 512):
        z = st.logits[r:r + 512].double()
        lp = torch.log_softmax(z, -1)
        parts[0].append(lp.gather(1, st.targets[r:r + 512].long()[:, None])[:, 0])
        parts[1].append(-torch.xlogy(lp.exp(), lp.exp()).sum(-1))
        order = torch.sort(z, dim=-1, descending=True, stable=True).indices[:, :st.top]
        parts[2].append(lp.gather(1, order))
        ids.append(order.to(torch.int32))
    return [torch.cat(parts[0]), torch.cat(parts[1]), torch.cat(ids), torch.cat(parts[2])]
