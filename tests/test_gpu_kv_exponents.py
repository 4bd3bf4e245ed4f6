"""Scale exponents at the ends of their byte: 0 stands for a scale of 0, 254 for 2^127, 255 for no
number, in single rows and in chunks alike.  Tolerances as tests/test_gpu_kv_attention.py
derives them."""
import numpy as np
import pytest
import torch

from tests._step import DeviceCache, device_rows, shape
from tests.test_gpu_kv_nonfinite import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("memory", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("size", [("slot", 256, [200], [0, 1], 1), ("head", 256, [150], [0, 5], 5),
                                  ("paged", 512, [300], [0, 100], 100)])
@pytest.mark.parametrize("name,e", [("v", 0), ("v", 255), ("k", 0), ("k", 255)])
def test_ends_of_the_exponents(name, e, size, dtype, memory):
    """One head's block of the memory."""
    c = Case(8, 2, 64, *size, dtype, seed=e)
    c.exps[name][0, 3, 1] = e
    if e == 0 and name == "v":   # (no value to hide behind: what is left is that block's alone)
        c.exps["v"][0, :, 1] = 0
    got, ls, want = c.run(memory)
    if name == "v":
        assert (got[:, 4:] == 0).all() if e == 0 else got[:, 4:].isnan().all()
    c.check(got, ls, want)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("count", [6, 100])
def test_a_new_block_of_no_numbers(count, dtype):
    """An exponent of 255 over the values of new tokens reaches the rows that see them and no others."""
    c = Case(8, 2, 64, "slot", 512, [318], [0, count], count, dtype)
    c.exps["v"][0, 10, 0] = 255   # slots 320 .. 351
    got, ls, want = c.run()
    assert got[:2].isfinite().all() and got[2:, :4].isnan().all()
    c.check(got, ls, want)


@pytest.mark.parametrize("e_old", [0, 254, 255])
def test_append_to_a_block_whose_scale_is_at_an_end(e_old):
    """Older codes under a scale of 0 are 0 in the larger one; a scale of 2^127 takes values near the
    end of fp32; where the scale is no number nothing becomes one."""
    import paper_2607_27600_gb300 as pkg
    from paper_2607_27600_gb300 import cc
    s, cap, block = shape(2, 1, 64), 64, 32
    codes = {n: np.full((1, cap, 1, 64), 0x7E, np.uint8) for n in "kv"}   # 448
    exps = {n: np.full((1, 2, 1), e_old, np.uint8) for n in "kv"}
    c = DeviceCache(pkg, codes, exps, [10], "slot")
    x = torch.full((1, 1, 64), {0: 2.0 ** -116, 254: 2.0 ** 125, 255: 1.0}[e_old], device="cuda")
    cc.cc_kv_append(s, c.cache, 0, device_rows(pkg, [1]), x, x, rotate=False)
    assert cc.cc_get_status() == cc.CC_OK
    for n in "kv":
        e, new, old = int(c.get(n + "_exp")[0, 0, 0]), c.get(n)[0, 10], c.get(n)[0, :10]
        if e_old == 0:
            assert e == 10 and (old == 0).all()
            # 2^-116 under a scale of 2^-117
            assert (new == 0x40).all()
        elif e_old == 254:
            assert e == 254 and (old == 0x7E).all()
            assert (new == 0x28).all()   # 2^125 / 2^127
        else:
            assert e == 255
