"""Pins of the oracle of the cache's management (oracle/step.py: received,
compact_blocks, join_parts): closed forms and library routines (CPU)."""
import numpy as np
import pytest
import torch

import oracle
from tests._step import quantised, starts, values


def case(seed, hq=4, hkv=2, dh=8, lens=(5, 0, 9), counts=(2, 3, 1), cap=16):
    rng = np.random.default_rng(seed)
    k = rng.standard_normal((len(lens), cap, hkv, dh))
    q = rng.standard_normal((sum(counts), hq, dh))
    return q, k, list(lens), starts(counts)


@pytest.mark.parametrize("memory", [False, True])
def test_received_weights_of_a_row_sum_to_one(memory):
    q, k, lens, start = case(1)
    _, lse, _ = oracle.attend_rows(q, k, k, lens, start, memory)
    got, slack = oracle.received(q, k, lse, lens, start, memory)
    seen = [(start[b + 1] - start[b]) * q.shape[1] * (lens[b] > 0 or not memory) for b in range(len(lens))]
    np.testing.assert_allclose(got.sum(1), seen, rtol=1e-12)
    assert (slack >= got * 0).all()
    for b, (n, m) in enumerate(zip(lens, np.diff(start))):
        assert not got[b, n + (0 if memory else m):].any()


def test_received_is_the_softmaxs_column_sums():
    q, k, lens, start = case(2, lens=(7,), counts=(1,))
    _, lse, _ = oracle.attend_rows(q, k, k, lens, start)
    want = torch.zeros(8, dtype=torch.float64)
    for h in range(4):
        want += torch.softmax(torch.from_numpy(k[0, :8, h // 2] @ q[0, h]) / 8 ** 0.5, 0)
    np.testing.assert_allclose(oracle.received(q, k, lse, lens, start)[0][0, :8], want.numpy(), rtol=1e-12)


def test_received_of_equal_keys_and_of_no_lse():
    q, k, lens, start = case(3, lens=(3,), counts=(1,))
    k[:] = 1.0
    _, lse, _ = oracle.attend_rows(q, k, k, lens, start)
    got, _ = oracle.received(q, k, lse, lens, start)
    np.testing.assert_allclose(got[0, :4], 1.0, rtol=1e-12)   # four heads, four slots
    for none in (-np.inf, np.inf, np.nan):
        lse[0, 1] = none
        np.testing.assert_allclose(oracle.received(q, k, lse, lens, start)[0][0, :4], 0.75, rtol=1e-12)


def test_compaction_of_one_scale_is_a_gather():
    rng = np.random.default_rng(4)
    codes, exps = quantised(rng, 2, 64, 2, 8, 16)
    exps[:] = 120
    keep = [np.sort(rng.choice(60, 21, False)), np.arange(0)]
    c, e = oracle.compact_blocks(codes, exps, 16, keep)
    np.testing.assert_array_equal(c[0, :21], codes[0, keep[0]])
    np.testing.assert_array_equal(c[0, 21:], codes[0, 21:])
    np.testing.assert_array_equal(c[1], codes[1])
    assert (e == 120).all()


def test_compaction_rounds_to_the_largest_scale():
    rng = np.random.default_rng(5)
    codes, exps = quantised(rng, 1, 128, 3, 8, 16, (1e-4, 10.0))
    keep = [np.sort(rng.choice(128, 50, False))]
    c, e = oracle.compact_blocks(codes, exps, 16, keep)
    old, new = values(codes, exps)[0, keep[0]], values(c, e)[0, :50]
    top = np.repeat(e[0, :4].astype(int), 16, 0)[:50]
    assert all(top[i, g] == exps[0, keep[0][i // 16 * 16:i // 16 * 16 + 16] // 16, g].max()
               for i in range(50) for g in range(3))
    # half a step: 2^-4 of a value, or of the least normal one
    floor = 2.0 ** (top - 127.0 - 6)
    assert (np.abs(new - old) <= 2.0 ** -4 * np.maximum(np.abs(old), floor[..., None])).all()


def test_compaction_of_scales_that_are_none():
    codes = np.full((1, 32, 1, 2), 0x38, np.uint8)   # 1.0
    codes[0, 1, 0, 1] = 0x7F
    exps = np.array([[[255], [127]]], np.uint8)
    c, e = oracle.compact_blocks(codes, exps, 16, [[1, 20]])
    assert e[0, 0, 0] == 127 and (c[0, 0] & 0x7F == 0x7F).all() and (c[0, 1] == 0x38).all()
    c, e = oracle.compact_blocks(codes, exps, 16, [[1, 3]])
    assert e[0, 0, 0] == 255 and c[0, 0, 0, 0] == 0x38
    exps[:] = [[[0], [100]]]
    c, e = oracle.compact_blocks(codes, exps, 16, [[1, 20]])
    assert e[0, 0, 0] == 100 and c[0, 0, 0, 0] == 0 and c[0, 0, 0, 1] == 0x7F and c[0, 1, 0, 0] == 0x38


def test_parts_joined_are_the_whole():
    q, k, lens, _ = case(6, lens=(12,), counts=(1,))
    rng = np.random.default_rng(7)
    v = rng.standard_normal(k.shape)
    start = starts([1])
    out, lse, _ = oracle.attend_rows(q, k, v, lens, start, True)
    a = oracle.attend_rows(q, k[:, :5], v[:, :5], [5], start, True)[:2]
    b = oracle.attend_rows(q, k[:, 5:12], v[:, 5:12], [7], start, True)[:2]
    none = np.full_like(out, np.nan), np.full_like(lse, -np.inf)
    got, s = oracle.join_parts([a[0], none[0], b[0]], [a[1], none[1], b[1]])
    np.testing.assert_allclose(got, out, rtol=1e-12)
    np.testing.assert_allclose(s, lse, rtol=1e-12)
    got, s = oracle.join_parts([none[0]] * 2, [none[1]] * 2)
    assert (got == 0).all() and (s == -np.inf).all()
    got, s = oracle.join_parts([a[0], b[0]], [a[1], b[1] * np.inf])
    assert (got == 0).all() and np.isnan(s).all()
