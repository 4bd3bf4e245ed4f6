"""cc_token_logprobs against the fp64 oracle (oracle/step.py): types, vocabularies
from one id to one that fills clusters of CTAs, odd pitches, ties, forbidden ids,
the types' lowest value as a mask, and what is no number.

Tolerances: fp32 sums of a few hundred terms a thread, joined pairwise: 2^-20
relative of S and W, so 2^-19 of the size of what they give (ln S, W / S <= ln
vocab < 13), and the subtraction z - m - ln S: 2^-22 of the result's size."""
import numpy as np
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module")
def cc():
    from paper_2607_27600_gb300 import cc as m
    m.load_library()
    return m


def answer(cc, z, targets, top, stream=None):
    n = z.shape[0]
    lp, ent = torch.full((n,), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
    ids = torch.full((n, top), -9, dtype=torch.int32, device="cuda") if top else None
    tlp = torch.full((n, top), 7.0, device="cuda") if top else None
    cc.cc_token_logprobs(z, targets, lp, ent, ids, tlp, stream)
    return [None if x is None else x.cpu().numpy() for x in (lp, ent, ids, tlp)]


def laid_out(z, dtype, pad):
    buf = torch.full((z.shape[0], z.shape[1] + pad), float("nan"), dtype=dtype, device="cuda")
    buf[:, :z.shape[1]] = torch.from_numpy(z).to(dtype).cuda()
    return buf[:, :z.shape[1]]


def check(got, want, z):
    lp, ent, ids, tlp = got
    close = 2.0 ** -19 * 13
    for g, w in ((lp, want[0]), (ent, want[1]), (tlp, want[3])):
        if g is None:
            continue
        f = np.isfinite(w)
        np.testing.assert_array_equal(g[~f], w[~f])
        assert (np.abs(g - w)[f] <= close + 2.0 ** -22 * np.abs(w[f])).all(), np.abs(g - w)[f].max()
    if ids is not None:
        np.testing.assert_array_equal(ids, want[2])


CASES = [
    # rows, vocab, dtype, top, pad, spread of the logits
    (3, 1, "f32", 1, 0, 2.0), (2, 2, "bf16", 2, 3, 2.0), (5, 7, "bf16", 7, 0, 2.0), (4, 8, "f16", 0, 0, 2.0),
    (3, 31, "f32", 31, 1, 2.0), (9, 33, "bf16", 32, 5, 2.0), (2, 511, "f16", 32, 1, 2.0),
    (3, 4095, "bf16", 20, 1, 3.0), (3, 4097, "f32", 32, 0, 3.0), (2, 8193, "bf16", 5, 7, 3.0),
    (1, 32768, "bf16", 32, 0, 2.0), (1, 50257, "f32", 20, 0, 3.0), (77, 32003, "f16", 3, 0, 1.0),
    (40, 65537, "bf16", 32, 0, 3.0), (160, 20011, "f32", 1, 0, 3.0), (400, 9999, "bf16", 8, 1, 30.0),
]


@pytest.mark.parametrize("rows,vocab,dtype,top,pad,spread", CASES)
def test_matches_oracle(cc, rows, vocab, dtype, top, pad, spread):
    rng = np.random.default_rng(vocab)
    z = torch.from_numpy(rng.standard_normal((rows, vocab)) * spread).to(TYPES[dtype]).double().numpy()
    t = rng.integers(0, vocab, rows).astype(np.int32)
    got = answer(cc, laid_out(z, TYPES[dtype], pad), torch.from_numpy(t).cuda(), top)
    assert cc.cc_get_status() == cc.CC_OK
    check(got, oracle.token_logprobs(z, t, top), z)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_ties_masks_and_order(cc, dtype):
    """Equal logits, rounded ones, ascending and descending ones (every thread's last or first
    is its largest), all but a few forbidden, a mask of the type's lowest value,
    zeros of both signs."""
    vocab, low = 9001, float(torch.finfo(TYPES[dtype]).min)
    rng = np.random.default_rng(1)
    z = np.zeros((10, vocab))
    z[1] = 3.25
    z[2] = np.round(rng.standard_normal(vocab))
    z[3] = np.arange(vocab) / 300.0
    z[4] = -np.arange(vocab) / 300.0
    z[5] = -np.inf
    z[5, [17, 4000, 8999, 5]] = [1.0, 2.0, 1.0, -3.0]
    z[6] = low
    z[6, rng.integers(0, vocab, 50)] = rng.standard_normal(50)
    z[7] = low
    z[8] = np.where(rng.random(vocab) < 0.5, 0.0, -0.0)
    z[9] = np.repeat(np.arange(vocab // 1000 + 1), 1000)[:vocab]
    z = torch.from_numpy(z).to(TYPES[dtype]).double().numpy()
    t = np.array([0, 9000, 5, 1, 2, 4000, 3, 8, 9, 0], np.int32)
    got = answer(cc, laid_out(z, TYPES[dtype], 0), torch.from_numpy(t).cuda(), 32)
    assert cc.cc_get_status() == cc.CC_OK
    want = oracle.token_logprobs(z, t, 32)
    # (relative to the lowest fp32, ln vocab is lost in z - lse but not in (z - m) - ln S)
    check(got, want, z)


def test_targets(cc):
    """-1 is no target; one outside the vocabulary is reported; a forbidden one is -inf."""
    z = torch.randn(5, 300, device="cuda")
    z[3, 7] = -float("inf")
    t = torch.tensor([0, -1, 299, 7, 12], dtype=torch.int32, device="cuda")
    lp = answer(cc, z, t, 0)[0]
    assert cc.cc_get_status() == cc.CC_OK
    want = torch.log_softmax(z.double(), -1).cpu().numpy()
    assert lp[1] == 0 and lp[3] == -np.inf
    assert np.abs(lp[[0, 2, 4]] - want[[0, 2, 4], [0, 299, 12]]).max() < 1e-5
    for bad in (300, -2):
        t[2] = bad
        lp2 = answer(cc, z, t, 0)[0]
        assert cc.cc_get_status() == cc.CC_ERR_DEVICE_ARG
        assert lp2[2] == 0 and (lp2[[0, 1, 3, 4]] == lp[[0, 1, 3, 4]]).all()


@pytest.mark.parametrize("rows", [5, 700])
def test_not_a_number(cc, rows):
    """Rows that allow nothing or hold NaN or +inf: NaN, with ids by what can be ordered;
    their neighbours are right."""
    vocab = 20000
    rng = np.random.default_rng(2)
    z = rng.standard_normal((rows, vocab)).astype(np.float32)
    clean = z.astype(np.float64).copy()
    z[1] = -np.inf
    z[2, 11000], z[3, 3] = np.nan, np.inf
    t = np.zeros(rows, np.int32)
    lp, ent, ids, tlp = answer(cc, torch.from_numpy(z).cuda(), torch.from_numpy(t).cuda(), 6)
    assert cc.cc_get_status() == cc.CC_OK
    want = oracle.token_logprobs(clean, t, 6)
    ok = np.array([r for r in range(rows) if r not in (1, 2, 3)])
    check([lp[ok], ent[ok], ids[ok], tlp[ok]], [w[ok] for w in want], z)
    for r in (1, 2, 3):
        assert np.isnan(lp[r]) and np.isnan(ent[r]) and np.isnan(tlp[r]).all()
    assert ids[1].tolist() == list(range(6)) and ids[3][0] == 3
    order = np.lexsort((np.arange(vocab), -np.where(np.isnan(z[2]), -np.inf, z[2])))
    assert ids[2].tolist() == order[:6].tolist()


def test_some_outputs_alone_and_another_stream(cc):
    z = torch.randn(3, 40000, device="cuda")
    t = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    whole = answer(cc, z, t, 4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ids, ent = torch.empty(3, 4, dtype=torch.int32, device="cuda"), torch.empty(3, device="cuda")
    cc.cc_token_logprobs(z, top_ids=ids, stream=side)
    cc.cc_token_logprobs(z, entropy=ent, stream=side)
    assert cc.cc_get_status(side) == cc.CC_OK
    assert (ids.cpu().numpy() == whole[2]).all() and (ent.cpu().numpy() == whole[1]).all()
