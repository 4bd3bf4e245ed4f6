"""Pins of the serving step's oracle (oracle/step.py): library routines, closed
forms and values the definitions name (CPU)."""
import numpy as np
import pytest
import scipy.stats
import torch

import oracle
from oracle.step import E_MAX, E_MIN
from synth.configs import ModelShape

SHAPE = ModelShape(1, 256, 4, 2, 64, 384, 100, 1e4, 1e-5)


def test_rotation_is_the_refreshs():
    x = np.random.default_rng(0).standard_normal((5, 4, 64))
    pos = np.array([0, 1, 77, 4096, 131071])
    np.testing.assert_allclose(oracle.rotate_rows(SHAPE, x, pos), oracle.rope(x, pos, SHAPE.rope_theta),
                               rtol=0, atol=1e-12)


@pytest.mark.parametrize("bound,e", [(448.0, 127), (448.0001, 128), (224.0, 126), (1.75, 119), (1.0, 119),
                                     (1.7501, 120), (0.0, 0), (1e-40, E_MIN), (3e38, 247), (2.0 ** 127, 246)])
def test_block_exponent(bound, e):
    assert oracle.block_exponent(bound) == min(e, E_MAX)
    if 0 < bound and E_MIN < e < E_MAX:
        assert bound <= 448 * 2.0 ** (e - 127) and bound > 448 * 2.0 ** (e - 128)


def test_pair_bound_holds_for_every_angle():
    rng = np.random.default_rng(1)
    k = rng.standard_normal((50, 2, 64)) * 10.0 ** rng.uniform(-3, 3, (50, 2, 64))
    top = max(np.abs(oracle.rotate_rows(SHAPE, k, np.full(50, p))).max(-1).max() for p in range(0, 3000, 7))
    assert top <= oracle.k_bound(k).max() * (1 + 1e-6)
    radius = np.hypot(k[..., :32], k[..., 32:]).max(-1)
    assert (oracle.k_bound(k) >= radius * (1 - 1e-6)).all() and (oracle.k_bound(k) <= radius * 1.119).all()


def blocks(rng, b, cap, block, h, dh):
    return (rng.integers(0, 256, (b, cap, h, dh)).astype(np.uint8),
            rng.integers(0, 256, (b, cap // block, h)).astype(np.uint8))


def test_append_one_at_a_time_and_all_at_once():
    """Rows of falling magnitude: the exponents never grow after the first row
    of a block, so the order of appending changes nothing."""
    rng = np.random.default_rng(2)
    codes, exps = blocks(rng, 1, 64, 16, 2, 8)
    x = rng.uniform(1, 2, (40, 2, 8)) * (2.0 ** -np.arange(40))[:, None, None]
    bound = np.abs(x).max(-1)
    # (an older slot decides the first block's exponent: make it small)
    exps[0, 0] = 20
    whole = oracle.append_blocks(codes, exps, 16, [3], [0, 40], x, bound)
    c, e = codes, exps
    for i in range(40):
        c, e, _ = oracle.append_blocks(c, e, 16, [3 + i], [0, 1], x[i:i + 1], bound[i:i + 1])
    np.testing.assert_array_equal(c, whole[0])
    np.testing.assert_array_equal(e, whole[1])


def test_append_scalar_case():
    """Block of 16, one head: values 1 and -3 (e: 448 * 2^-7 = 3.5 holds 3), then 100
    (448 * 2^-2 = 112): the old codes are rescaled by 2^-5."""
    codes, exps = np.zeros((1, 16, 1, 2), np.uint8), np.full((1, 1, 1), 250, np.uint8)
    x = np.array([[[1.0, -3.0]]])
    c, e, _ = oracle.append_blocks(codes, exps, 16, [0], [0, 1], x, np.array([[3.0]]))
    assert e[0, 0, 0] == 120 and oracle.e4m3_decode(c[0, 0, 0]).tolist() == [128.0, -384.0]
    c, e, _ = oracle.append_blocks(c, e, 16, [1], [0, 1], np.array([[[100.0, 0.0]]]), np.array([[100.0]]))
    assert e[0, 0, 0] == 125
    # 400 lies between 384 and 416: the even code
    assert (oracle.e4m3_decode(c[0, :2, 0]) * 0.25).tolist() == [[1.0, -3.0], [96.0, 0.0]]
    # zeros alone: any scale holds them, the older slots keep theirs
    c2, e2, _ = oracle.append_blocks(c, e, 16, [2], [0, 1], np.zeros((1, 1, 2)), np.zeros((1, 1)))
    assert e2[0, 0, 0] == 125 and (c2[0, :2] == c[0, :2]).all()
    _, e3, _ = oracle.append_blocks(codes, exps, 16, [0], [0, 1], np.zeros((1, 1, 2)), np.zeros((1, 1)))
    assert e3[0, 0, 0] == 127


def test_written_values_are_within_half_a_step():
    rng = np.random.default_rng(3)
    codes, exps = blocks(rng, 2, 64, 32, 2, 16)
    x = rng.standard_normal((50, 2, 16))
    start, seq = [0, 30, 50], [17, 40]
    exps[:] = 118
    c, e, exact = oracle.append_blocks(codes, exps, 32, seq, start, x, np.abs(x).max(-1))
    scale = 2.0 ** (np.repeat(e.astype(int), 32, 1)[..., None] - 127)
    got = oracle.e4m3_decode(c) * scale
    w = ~np.isnan(exact)
    step = np.maximum(2.0 ** (np.floor(np.log2(np.abs(exact[w]))) - 3), (scale * 2.0 ** -9 + 0 * exact)[w])
    assert w.sum() == 50 * 32 and (np.abs(got[w] - exact[w]) <= step / 2 * (1 + 1e-12)).all()


@pytest.mark.parametrize("memory_only", [False, True])
def test_attention_is_sdpa(memory_only):
    rng = np.random.default_rng(4)
    q, start, seq = rng.standard_normal((7, 4, 16)), [0, 3, 3, 7], [5, 9, 0]
    k, v = rng.standard_normal((2, 3, 12, 2, 16))
    out, lse, _ = oracle.attend_rows(q, k, v, seq, start, memory_only)
    for b in range(3):
        m = start[b + 1] - start[b]
        if m == 0 or (memory_only and seq[b] == 0):
            assert (out[start[b]:start[b + 1]] == 0).all() and np.isinf(lse[start[b]:start[b + 1]]).all()
            continue
        end = seq[b] if memory_only else seq[b] + m
        mask = np.ones((m, end), bool) if memory_only else np.arange(end) <= seq[b] + np.arange(m)[:, None]
        t = [torch.from_numpy(x).transpose(0, 1) for x in (q[start[b]:start[b + 1]], k[b, :end].repeat(2, 1),
                                                           v[b, :end].repeat(2, 1))]
        want = torch.nn.functional.scaled_dot_product_attention(*t, attn_mask=torch.from_numpy(mask))
        np.testing.assert_allclose(out[start[b]:start[b + 1]], want.transpose(0, 1).numpy(), atol=1e-12)
        s = torch.matmul(t[0], t[1].transpose(-1, -2)) / 4
        want = torch.logsumexp(s.masked_fill(~torch.from_numpy(mask), -np.inf), -1).T.numpy()
        np.testing.assert_allclose(lse[start[b]:start[b + 1]], want, atol=1e-12)


def test_token_logprobs_are_log_softmax():
    rng = np.random.default_rng(5)
    z = rng.standard_normal((4, 300)) * 3
    z[1, ::3] = -np.inf
    z[2] = np.round(z[2])            # ties
    t = np.array([4, 7, 0, 299])
    lp, ent, ids, tlp = oracle.token_logprobs(z, t, 9)
    want = torch.log_softmax(torch.from_numpy(z), -1).numpy()
    np.testing.assert_allclose(lp, want[np.arange(4), t], atol=1e-12)
    np.testing.assert_allclose(ent, scipy.stats.entropy(np.exp(want), axis=-1), atol=1e-12)
    np.testing.assert_allclose(tlp, torch.topk(torch.from_numpy(want), 9).values.numpy(), atol=1e-12)
    for r in range(4):
        assert (np.diff(z[r][ids[r]]) <= 0).all()
        same = np.diff(z[r][ids[r]]) == 0
        assert (np.diff(ids[r])[same] > 0).all()
