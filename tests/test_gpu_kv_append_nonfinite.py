"""cc_kv_append of 16-bit rows with infinities and NaN among them: no part in the exponents, NaN codes
where they land, everything else as without them.  (fp32 rows: tests/test_gpu_kv_append.py.)"""
import numpy as np
import pytest
import torch

import oracle
from tests._step import DeviceCache, columns, device_rows, quantised, shape, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("count", [1, 3, 70])
def test_16_bit_rows(count, dtype):
    import paper_2607_27600_gb300 as pkg
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(count)
    s, cap, block, lens = shape(4, 2, 64), 128, 32, [20, 40]
    codes, exps = {}, {}
    for n in "kv":
        codes[n], exps[n] = quantised(rng, 2, cap, 2, 64, block)
    counts = [count, 2]
    k, v = (torch.from_numpy(rng.standard_normal((sum(counts), 2, 64)) * 3).to(dtype).double().numpy()
            for _ in range(2))
    for i, x in enumerate((np.inf, -np.inf, np.nan)):
        r = i % count   # of sequence 0; head 1 of the values is left alone
        k[r, i % 2, 5 * i], v[r, 0, 7 * i + 1] = x, x
    c = DeviceCache(pkg, codes, exps, lens, "slot")
    dk, dv = columns([k, v], dtype)
    cc.cc_kv_append(s, c.cache, 0, device_rows(pkg, counts), dk, dv, rotate=False)
    assert cc.cc_get_status() == cc.CC_OK
    for n, x, bound in (("k", k, oracle.k_bound(k)), ("v", v, oracle.v_bound(v))):
        wc, we, exact = oracle.append_blocks(codes[n], exps[n], block, lens, starts(counts), x, bound)
        np.testing.assert_array_equal(c.get(n + "_exp"), we)
        none = np.isnan(oracle.e4m3_decode(wc))
        assert none.sum() == 3
        np.testing.assert_array_equal(np.isnan(oracle.e4m3_decode(c.get(n))), none)
        np.testing.assert_array_equal(c.get(n)[~none], wc[~none])
