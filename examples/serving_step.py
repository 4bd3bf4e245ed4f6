"""Serving over an 8-bit K/V cache with the model's own projections.

    python examples/serving_step.py [--steps 16]

A small random decoder (the layer cc_append_chunk runs: RMSNorm, GQA attention
with rotate-half RoPE, SwiGLU) whose matrix products are this file's, in plain
torch.  The library holds the cache: per layer cc_kv_append writes the new tokens'
keys and values into a paged cache of e4m3 codes with a power-of-two scale for each
block of slots and KV head, cc_kv_attention reads it, and cc_token_logprobs answers
with each next token, how likely it was, and how sure the model is.  A prompt of
each sequence goes in as one chunk, then tokens one at a time.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_27600_gb300 as pkg  # noqa: E402
from paper_2607_27600_gb300 import cc  # noqa: E402
from synth.configs import ModelShape  # noqa: E402

SHAPE = ModelShape(n_layers=2, d_model=512, n_q_heads=8, n_kv_heads=2, head_dim=64, d_ff=1408,
                   vocab=4096, rope_theta=1e4, rms_eps=1e-5)
PAGE, BLOCK = 128, 32


class Model:
    """Random bf16 weights; q, k and v of a layer in one matrix."""

    def __init__(self, shape, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        s = self.shape = shape

        def w(*dims):
            return torch.randn(dims, generator=g, device="cuda").mul_(0.02).to(torch.bfloat16)

        qkv = (s.n_q_heads + 2 * s.n_kv_heads) * s.head_dim
        self.embed, self.lm_head = w(s.vocab, s.d_model), w(s.vocab, s.d_model)
        self.layers = [{"qkv": w(qkv, s.d_model), "o": w(s.d_model, s.n_q_heads * s.head_dim),
                        "gate_up": w(2 * s.d_ff, s.d_model), "down": w(s.d_model, s.d_ff)}
                       for _ in range(s.n_layers)]

    def norm(self, h):
        return (h * torch.rsqrt(h.square().mean(-1, keepdim=True) + self.shape.rms_eps)).to(torch.bfloat16)


def empty_cache(shape, batch, cap):
    """A paged block-format cache; pages in any order."""
    s, pages = shape, batch * cap // PAGE
    table = torch.randperm(pages, device="cuda").to(torch.int32).view(batch, -1).contiguous()

    def pools(*dims):
        return [torch.zeros(dims, dtype=torch.uint8, device="cuda") for _ in range(s.n_layers)]

    return pkg.Cache({
        "k": pools(pages, PAGE, s.n_kv_heads, s.head_dim), "v": pools(pages, PAGE, s.n_kv_heads, s.head_dim),
        "k_exp": pools(pages, PAGE // BLOCK, s.n_kv_heads), "v_exp": pools(pages, PAGE // BLOCK, s.n_kv_heads),
        "kv_block": BLOCK, "block_table": table, "page_size": PAGE,
        "seq_len": torch.zeros(batch, dtype=torch.int32, device="cuda"),
        "tokens": torch.zeros(batch, cap, dtype=torch.int32, device="cuda"),
        "pos": torch.zeros(batch, cap, dtype=torch.int32, device="cuda")})


def step(model, cache, rows, tokens, last, top=4):
    """Runs the rows' tokens (int32 [n]) through every layer and the cache, and
    answers from the rows `last` (the last one of each sequence): the `top` most
    likely next tokens, their log-probabilities and the entropy."""
    s, n = model.shape, len(tokens)
    cfg = cc.model_cfg(s)
    q_dim, kv_dim = s.n_q_heads * s.head_dim, s.n_kv_heads * s.head_dim
    ws = cc.alloc_workspace(cc.cc_kv_attention_workspace_size(cfg, cache, rows))
    q = torch.empty(n, s.n_q_heads, s.head_dim, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    h = model.embed[tokens.long()].float()
    for l, w in enumerate(model.layers):
        qkv = model.norm(h) @ w["qkv"].T
        # q, k and v are columns of one product; the library takes them where they lie
        k = qkv[:, q_dim:q_dim + kv_dim].view(n, s.n_kv_heads, s.head_dim)
        v = qkv[:, q_dim + kv_dim:].view(n, s.n_kv_heads, s.head_dim)
        cc.cc_kv_append(cfg, cache, l, rows, k, v, qkv[:, :q_dim].view_as(q), q)
        cc.cc_kv_attention(cfg, cache, l, rows, q, out, ws)
        h = h + (out.view(n, q_dim) @ w["o"].T).float()
        gate, up = (model.norm(h) @ w["gate_up"].T).chunk(2, -1)
        h = h + ((torch.nn.functional.silu(gate) * up) @ w["down"].T).float()
    cc.cc_kv_advance(cache, rows, tokens)
    logits = model.norm(h[last]) @ model.lm_head.T
    b = len(last)
    ids = torch.empty(b, top, dtype=torch.int32, device="cuda")
    lp, ent = torch.empty(b, top, device="cuda"), torch.empty(b, device="cuda")
    cc.cc_token_logprobs(logits, entropy=ent, top_ids=ids, top_logprob=lp)
    return ids, lp, ent


def serve(prompts, steps, cap=512, seed=0, chunked=True):
    """Greedy continuations of the prompts (lists of token ids): ids [b, steps + 1],
    log-probabilities and entropies of the same shape, and the cache.  chunked:
    whole prompts at once, else token by token (prompts of one length)."""
    model, b = Model(SHAPE, seed), len(prompts)
    cache = empty_cache(SHAPE, b, cap)
    one = pkg.Rows(b)   # a row per sequence, at the positions that follow
    each = torch.arange(b, device="cuda")
    if chunked:
        start = torch.tensor([sum(map(len, prompts[:i])) for i in range(b + 1)], dtype=torch.int32, device="cuda")
        rows = pkg.Rows(sum(map(len, prompts)), start, max_rows=max(map(len, prompts)))
        flat = torch.tensor([t for p in prompts for t in p], dtype=torch.int32, device="cuda")
        ids, lp, ent = step(model, cache, rows, flat, start[1:].long() - 1)
    else:
        for column in torch.tensor(prompts, dtype=torch.int32, device="cuda").T.contiguous():
            ids, lp, ent = step(model, cache, one, column, each)
    answers = [(ids[:, 0], lp[:, 0], ent)]
    for _ in range(steps):
        ids, lp, ent = step(model, cache, one, answers[-1][0].contiguous(), each)
        answers.append((ids[:, 0], lp[:, 0], ent))
    if cc.cc_get_status() != cc.CC_OK:
        raise RuntimeError("a step reported a device-side error")
    return [torch.stack(x, 1) for x in zip(*answers)] + [cache]


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=16)
    steps = ap.parse_args().steps
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, SHAPE.vocab, (n,), generator=g).tolist() for n in (200, 33, 1)]
    ids, lp, ent, cache = serve(prompts, steps)
    for i, p in enumerate(prompts):
        print(f"sequence {i}: prompt of {len(p)}, {int(cache.d['seq_len'][i])} slots, mean log-probability "
              f"{float(lp[i].mean()):.3f}, mean entropy {float(ent[i].mean()):.3f}, next {ids[i].tolist()}")


if __name__ == "__main__":
    main()
