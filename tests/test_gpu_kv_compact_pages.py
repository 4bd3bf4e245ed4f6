"""cc_kv_compact where a page lies outside the pool, exactly: slots that come from it keep
their values beside slots that move into their block, slots that would go to it are not
written, and the other sequence's results stand."""
import numpy as np
import pytest

import oracle
from tests.test_gpu_kv_compact import Case, pkg  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("stds", [(0.5, 2.0), (0.002, 500.0)])
@pytest.mark.parametrize("block", [16, 64, 128])
@pytest.mark.parametrize("page", [0, 1, 2, 3])
def test_a_page_that_is_none(pkg, page, block, stds):  # noqa: F811
    from paper_2607_27600_gb300 import cc
    c = Case(pkg, 20 + page, 1, 2, 64, block, "paged", 512, [512, 500], [200, 150], stds=stds)
    before = {n: (c.get(n, 0), c.get(n + "_exp", 0)) for n in "kv"}
    c.c.d["block_table"][0, page] = c.c.n_pages if page % 2 else -1
    assert c.run() == cc.CC_ERR_DEVICE_ARG
    # a slot that comes from the page is its own source
    src = np.where(c.keep[0] // 128 == page, np.arange(len(c.keep[0])), c.keep[0])
    moved = (src != np.arange(len(src)))
    assert any(0 < moved[j:j + block].sum() < len(moved[j:j + block]) for j in range(0, len(src), block))
    lo, hi = 128 * page, min(128 * page + 128, len(src))   # slots that would go to it
    for n in "kv":
        codes, exps = oracle.compact_blocks(c.codes[0][n], c.exps[0][n], block, [src, c.keep[1]])
        codes[0, lo:hi], exps[0, lo // block:-(-hi // block)] = before[n][0][0, lo:hi], before[n][1][0, lo // block:-(-hi // block)]
        np.testing.assert_array_equal(c.get(n + "_exp", 0), exps)
        got = c.get(n, 0)
        nan = (codes & 0x7F) == 0x7F
        np.testing.assert_array_equal((got & 0x7F) == 0x7F, nan)
        np.testing.assert_array_equal(np.where(nan, 0, got), np.where(nan, 0, codes))
    # what the pages do not hold moves all the same
    for n, x in c.small.items():
        want = x.copy()
        for i, k in enumerate(c.keep):
            want[i, :len(k)] = x[i, k]
        np.testing.assert_array_equal(c.c.d[n].cpu().numpy(), want)
    assert c.c.d["seq_len"].tolist() == [200, 150]
