"""examples/serving_step.py: the three operators together."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serving_step.py")
    spec = importlib.util.spec_from_file_location("serving_step", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def cached(cache, name, l, b, n):
    """Values of the first n slots of sequence b in layer l's pages."""
    d = cache.d
    slot = torch.arange(n, device="cuda")
    row = d["block_table"][b].long()[slot // d["page_size"]] * d["page_size"] + slot % d["page_size"]
    codes = d[name][l].flatten(0, 1)[row].view(torch.float8_e4m3fn).float()
    return codes * torch.exp2(d[name + "_exp"][l].flatten(0, 1)[row // d["kv_block"]].float() - 127)[..., None]


def dense(ex, prompts, steps_ids, cache):
    """Log-probabilities that the same model gives the ids [b][steps + 1] where its keys
    and values are those that the cache holds."""
    m, s = ex.Model(ex.SHAPE), ex.SHAPE
    g, out = s.n_q_heads // s.n_kv_heads, []
    half = s.head_dim // 2
    freq = s.rope_theta ** (-2.0 * torch.arange(half, device="cuda", dtype=torch.float64) / s.head_dim)

    def rope(x):
        ang = (torch.arange(x.shape[0], device="cuda", dtype=torch.float64)[:, None] * freq)[:, None]
        c, sn = ang.cos().float(), ang.sin().float()
        a, b = x[..., :half], x[..., half:]
        return torch.cat([a * c - b * sn, b * c + a * sn], -1)

    for i, (p, ids) in enumerate(zip(prompts, steps_ids)):
        seq = torch.tensor(p + ids[:-1], device="cuda")
        h, n = m.embed[seq].float(), len(seq)
        mask = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
        for l, w in enumerate(m.layers):
            qkv = (m.norm(h) @ w["qkv"].T).float().view(n, -1, s.head_dim)
            q, k, v = qkv.split([s.n_q_heads, s.n_kv_heads, s.n_kv_heads], 1)
            q, k = rope(q), rope(k)
            for name, x in (("k", k), ("v", v)):   # an e4m3 rounding away from what was appended
                held = cached(cache, name, l, i, n)
                assert ((held - x).abs() <= x.abs() * 2.0 ** -4 + x.abs().amax() * 2.0 ** -6).all()
            k, v = cached(cache, "k", l, i, n).repeat_interleave(g, 1), cached(cache, "v", l, i, n)
            sc = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(s.head_dim)
            a = torch.softmax(sc.masked_fill(~mask, -math.inf), -1)
            o = torch.einsum("hij,jhd->ihd", a, v.repeat_interleave(g, 1)).reshape(n, -1).to(torch.bfloat16)
            h = h + (o @ w["o"].T).float()
            gate, up = (m.norm(h) @ w["gate_up"].T).chunk(2, -1)
            h = h + ((torch.nn.functional.silu(gate) * up) @ w["down"].T).float()
        lp = torch.log_softmax((m.norm(h[len(p) - 1:]) @ m.lm_head.T).float(), -1)
        out.append(lp[torch.arange(len(ids)), torch.tensor(ids)])
    return torch.stack(out)


def test_steps_agree_with_a_dense_model(example):
    """Over the cache's own values what is left is bf16 rounding of activations (2^-8 of
    logits whose spread is 0.02 sqrt(512) = 0.45): well below 0.05."""
    g = torch.Generator().manual_seed(3)
    prompts = [torch.randint(0, example.SHAPE.vocab, (n,), generator=g).tolist() for n in (150, 40, 1)]
    ids, lp, ent, cache = example.serve(prompts, 6)
    assert cache.d["seq_len"].tolist() == [156, 46, 7]
    for i, p in enumerate(prompts):
        assert cache.d["tokens"][i, :len(p) + 6].tolist() == p + ids[i, :6].tolist()
        assert cache.d["pos"][i, :len(p) + 6].tolist() == list(range(len(p) + 6))
    assert ((ent > 0) & (ent <= math.log(example.SHAPE.vocab) + 1e-5)).all()
    want = dense(example, prompts, ids.tolist(), cache)
    assert (lp - want).abs().max() < 0.05


def test_chunk_and_single_tokens_agree(example):
    """One chunk of 70 tokens (the tile attention) or 70 steps: the caches differ by the
    codes that were rescaled on the way, the answers by as little as above."""
    g = torch.Generator().manual_seed(4)
    prompts = [torch.randint(0, example.SHAPE.vocab, (70,), generator=g).tolist() for _ in range(2)]
    one = example.serve(prompts, 0)
    many = example.serve(prompts, 0, chunked=False)
    assert (one[1] - many[1]).abs().max() < 0.05 and (one[2] - many[2]).abs().max() < 0.05
