"""cc_kv_accumulate of queries whose elements lie far apart, against the fp64 oracle.

Tolerances.  Those of test_gpu_kv_accumulate.py.  Single rows and few come to fp16 with the
largest element m of a row and head at 2^7 or above: an element is off by half of fp16's least step, 2^-25
there, at most, 2^-32 m.  A score is then off by d = 2^-32 m sum_i |K_i| / sqrt(head_dim), its weight
by a factor of e^d at most.  Chunks take the rows as they are (d = 0)."""
import numpy as np
import pytest
import torch

import oracle
from tests._step import DeviceCache, values
from tests.test_gpu_kv_accumulate import Case, pkg  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("counts", [[1, 1], [4, 9], [90, 70]])
@pytest.mark.parametrize("power", [12, 20, 24, 26])
@pytest.mark.parametrize("dh", [64, 128])
def test_one_element_far_above_the_others(pkg, dh, power, counts):  # noqa: F811
    """Its keys are 0, so that the score is the others'."""
    c = Case(pkg, power + dh, 8, 2, dh, 16, "slot", "bf16", 512, [200, 77], counts)
    c.q[..., 3] = 2.0 ** power * 1.5
    c.q[:, ::2, 3] *= -1
    c.codes["k"][..., 3] &= 0x80
    assert torch.equal(torch.from_numpy(c.q).to(c.t).double(), torch.from_numpy(c.q))
    c.k = values(c.codes["k"], c.exps["k"])
    _, lse, _ = oracle.attend_rows(c.q, c.k, c.k * 0, c.lens, c.start)
    c.lse = lse.astype(np.float32)
    c.c = DeviceCache(pkg, c.codes, c.exps, c.lens, "slot")
    want, tol = c.want()
    if max(counts) < 64:
        g = c.s.n_q_heads // c.s.n_kv_heads
        for b in range(2):
            for r in range(c.start[b], c.start[b + 1]):
                end = c.lens[b] + r - c.start[b] + 1
                for h in range(8):
                    x = c.k[b, :end, h // g]
                    w = np.exp(x @ c.q[r, h] / np.sqrt(dh) - float(c.lse[r, h]))
                    tol[b, :end] += w * np.expm1(2.0 ** -32 * np.abs(c.q[r, h]).max() * np.abs(x).sum(-1) / np.sqrt(dh))
    got = c.run()
    for b in range(2):
        end = c.ends[b]
        assert (np.abs(got - want)[b, :end] <= tol[b, :end]).all()


@pytest.mark.parametrize("dtype,spread", [("bf16", 40), ("f16", 28)])
@pytest.mark.parametrize("counts", [[1, 5], [80, 50]])
def test_elements_of_every_size(pkg, counts, dtype, spread):  # noqa: F811
    """Magnitudes even over their logarithm: the largest ones decide, the others' steps are below fp32's."""
    c = Case(pkg, 9, 8, 2, 64, 16, "paged", dtype, 512, [200, 77], counts)
    q = np.exp2(c.rng.uniform(3 - spread, 3, c.q.shape)) * c.rng.choice([-1.0, 1.0], c.q.shape)
    c.q = torch.from_numpy(q).to(c.t).double().numpy()
    _, lse, _ = oracle.attend_rows(c.q, c.k, c.k * 0, c.lens, c.start)
    c.lse = lse.astype(np.float32)
    c.check(c.run())
