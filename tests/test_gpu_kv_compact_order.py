"""cc_kv_compact where units wait for one another, exactly: sources, and exponents of blocks that
hold sources past the last kept slot, that a later chunk overwrites, over many layers."""
import numpy as np
import pytest

from tests.test_gpu_kv_compact import Case, pkg  # noqa: F401

pytestmark = pytest.mark.gpu


def keeps(n):
    """Keep-sets of n slots: chunk 0 reads from the block in which chunk 1 ends; the same from far behind;
    all but a few; one in a hundred left out."""
    return [np.r_[0:100, 200:228, n - 112:n - 100],
            np.r_[0:90, 250:256, 300:340, n - 30:n],
            np.r_[5:n],
            np.array([i for i in range(n) if i % 100])]


@pytest.mark.parametrize("layout,block,dh", [("slot", 128, 128), ("paged", 64, 64), ("head", 16, 128)])
def test_overwritten_by_later_chunks(pkg, layout, block, dh):  # noqa: F811
    from paper_2607_27600_gb300 import cc
    n = 1024
    c = Case(pkg, block, 6, 3, dh, block, layout, n, [n] * 4, keeps(n), h=False)
    for _ in range(5):
        c.build()
        assert c.run() == cc.CC_OK
        c.check()
