"""cc_kv_accumulate of chunks whose head group does not fill a tile of query rows: a slot
that is no number, seen only by rows without a finite lse, receives nothing from the tile
before these rows.  Against the fp64 oracle, with the tolerances of
test_gpu_kv_accumulate.py."""
import numpy as np
import pytest

from tests._step import DeviceCache, values
from tests.test_gpu_kv_accumulate import Case, pkg  # noqa: F401

pytestmark = pytest.mark.gpu

CASES = [
    # hq, hkv, dh, layout, lens, counts, the first row whose lse is not finite: in a tile's first place, or not
    (7, 1, 128, "slot", [0], [40], 13),
    (7, 1, 64, "paged", [3, 77], [60, 9], 26),
    (7, 1, 128, "head", [3], [40], 20),
    (14, 2, 128, "paged", [130, 0], [50, 40], 39),
    (5, 1, 64, "head", [3], [48], 19),
    (11, 1, 128, "slot", [100, 1], [30, 20], 16),
    (56, 1, 128, "paged", [77], [12], 5),
    (7, 1, 128, "slot", [20], [9], 4),   # (so few rows that there are no tiles)
]


def check(c, first):
    """Rows from `first` of sequence 0 on have no lse; the slots that only these see keep their totals."""
    c.lse[first:c.counts[0]] = np.nan
    c.lse[first:c.counts[0]:3] = -np.inf
    c.k = values(c.codes["k"], c.exps["k"])
    c.c = DeviceCache(c.pkg, c.codes, c.exps, c.lens, c.c.layout)
    n = c.lens[0] + first
    for zero in (False, True):
        got = c.run(first=zero)
        c.check(got, first=zero)
        own = c.lens[0] + c.counts[0]
        np.testing.assert_array_equal(got[0, n:own], c.acc[0, n:own] * (0 if zero else 1))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,dh,layout,lens,counts,first", CASES)
def test_codes_that_are_no_numbers(pkg, hq, hkv, dh, layout, lens, counts, first, dtype):  # noqa: F811
    c = Case(pkg, hq + first, hq, hkv, dh, 16, layout, dtype, 256, lens, counts)
    c.codes["k"][0, lens[0] + first, 0, 5] = 0x7F
    c.codes["k"][0, lens[0] + first, hkv - 1, dh - 1] = 0xFF
    check(c, first)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,lens,first", [(7, 3, 13), (7, 99, 13), (5, 13, 19), (56, 74, 6)])
def test_scales_that_are_none(pkg, hq, lens, first, dtype):  # noqa: F811
    """A block of exponent 255 that begins with the first such row's slot."""
    assert (lens + first) % 16 == 0
    c = Case(pkg, hq + lens, hq, 1, 128, 16, "slot", dtype, 256, [lens], [40])
    c.exps["k"][0, (lens + first) // 16] = 255
    check(c, first)
