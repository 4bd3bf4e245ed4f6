"""cc_kv_join against the fp64 oracle (oracle/step.py): types, head dims, pitches,
counts of parts, parts without slots, rows that failed, results in a part's place.

Tolerances.  A weight e^(s_i - m) carries the rounding of s_i - m and of the product with
log2 e, 2^-23 of it (|s_i - m| <= 40 where it counts), and a few units of fp32; the sums as
many as there are parts: 2^-17 of sum_i w_i |o_i| covers them.  The output is
rounded to its type (unit roundoff: bf16 2^-8, fp16 2^-11, fp32 2^-24; fp16 below 2^-14 lies
on a grid of 2^-24, so that half a step is 2^-25 there whatever the value); the lse is fp32."""
import numpy as np
import pytest
import torch

import oracle
from tests._step import columns, shape

pytestmark = pytest.mark.gpu
TYPES = {"bf16": (torch.bfloat16, 2.0 ** -8, 0), "f16": (torch.float16, 2.0 ** -11, 2.0 ** -25),
         "f32": (torch.float32, 2.0 ** -24, 0)}


@pytest.fixture(scope="module")
def pkg():
    import paper_2607_27600_gb300 as p
    p.load_library()
    return p


def draw(rng, t, k, n, hq, dh):
    parts = torch.from_numpy(rng.standard_normal((k, n, hq, dh))).to(t)
    lses = torch.from_numpy(rng.standard_normal((k, n, hq)) * 6 + 5).float()
    return parts, lses


def check(out, lse, parts, lses, eps, least):
    p, s = parts.double().numpy(), lses.double().numpy()
    want, want_lse = oracle.join_parts(p, s)
    spread, _ = oracle.join_parts(np.abs(p), s)
    got, ls = out.double().cpu().numpy(), lse.double().cpu().numpy()
    off = np.abs(got - want) / (eps * np.abs(want) + 2.0 ** -17 * spread + least + 1e-38)
    at = np.unravel_index(off.argmax(), off.shape)
    assert off[at] <= 1, (at, got[at], want[at], spread[at])
    f = np.isfinite(want_lse)
    np.testing.assert_array_equal(ls[~f], want_lse[~f])
    assert np.max(np.abs(ls[f] - want_lse[f]) - 2.0 ** -22 * np.abs(want_lse[f])) <= 2.0 ** -21


CASES = [(1, 1, 64, 1, 2, 0), (1, 7, 128, 1, 3, 0), (5, 8, 64, 2, 2, 8), (33, 28, 128, 4, 2, 0), (3, 3, 64, 3, 16, 24),
         (130, 12, 128, 2, 5, 0), (2, 5, 64, 5, 1, 16), (700, 32, 128, 8, 2, 0)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n,hq,dh,hkv,k,pad", CASES)
def test_matches_oracle(pkg, n, hq, dh, hkv, k, pad, dtype):
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(n * 100 + hq)
    t, *eps = TYPES[dtype]
    parts, lses = draw(rng, t, k, n, hq, dh)
    s = shape(hq, hkv, dh)
    # parts as columns of one buffer, the result in one with a pitch of its own
    at = columns([p.double().numpy() for p in parts], t, pad)
    wide = torch.full((n, hq * dh + 8), 7.0, dtype=t, device="cuda")
    out, lse = wide[:, :hq * dh].view(n, hq, dh), torch.full((n, hq), 7.0, device="cuda")
    cc.cc_kv_join(s, at, list(lses.cuda()), out, lse)
    check(out, lse, parts, lses, *eps)
    assert (wide[:, hq * dh:] == 7).all()
    again = torch.empty_like(out)
    cc.cc_kv_join(s, at, list(lses.cuda()), again)   # no lse; the same bits
    assert torch.equal(again, out)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_parts_without_slots_and_rows_that_failed(pkg, dtype):
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(9)
    t, *eps = TYPES[dtype]
    n, hq, dh, k = 40, 4, 64, 3
    parts, lses = draw(rng, t, k, n, hq, dh)
    lses[0, ::3] = -np.inf                       # these hold any bits
    parts[0, ::3] = float("nan")
    lses[:, 5, 1], lses[1, 7, 2], lses[2, 8, 3] = -np.inf, np.inf, np.nan
    lses[:, 9] += 3e38 / 8                       # far from each other, and large
    lses[:, 10] -= 1e5
    lses[1, 11] = lses[0, 11] - 300              # a weight that vanishes
    parts[:, 5, 1] = float("inf")
    out, lse = torch.empty(n, hq, dh, dtype=t, device="cuda"), torch.empty(n, hq, device="cuda")
    cc.cc_kv_join(shape(hq, 2, dh), list(parts.cuda()), list(lses.cuda()), out, lse)
    seen = torch.where(torch.isfinite(lses)[..., None], parts, torch.zeros((), dtype=t))   # (what is not looked at)
    check(out, lse, seen, lses, *eps)
    assert (out[5, 1] == 0).all() and float(lse[5, 1]) == -np.inf
    assert (out[7, 2] == 0).all() and torch.isnan(lse[7, 2]) and torch.isnan(lse[8, 3])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("place", [0, 1])
def test_in_a_parts_place(pkg, place, dtype):
    """out and lse where a part and its lse lie: the bits of a call with buffers of its own."""
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(10)
    t = TYPES[dtype][0]
    n, hq, dh = 333, 28, 128
    parts, lses = draw(rng, t, 2, n, hq, dh)
    p, s = list(parts.cuda()), list(lses.cuda())
    out, lse = torch.empty_like(p[0]), torch.empty_like(s[0])
    cc.cc_kv_join(shape(hq, 4, dh), p, s, out, lse)
    cc.cc_kv_join(shape(hq, 4, dh), p, s, p[place], s[place])
    assert torch.equal(p[place], out) and torch.equal(s[place], lse)


def test_refusals(pkg):
    from paper_2607_27600_gb300 import cc
    x, s = torch.zeros(4, 8, 64, device="cuda"), torch.zeros(4, 8, device="cuda")
    c = shape(8, 2, 64)
    for parts, lses, out in (([x[:3]], [s], x), ([x.half()], [s], x), ([x], [s[:3]], x), ([x], [s.half()], x),
                             ([x.transpose(1, 2)], [s], x), ([x], [s], x.transpose(1, 2))):
        with pytest.raises(ValueError):
            cc.cc_kv_join(c, parts, lses, out)
    with pytest.raises(cc.CCError):
        cc.cc_kv_join(c, [x] * 17, [s] * 17, x)
