"""cc_kv_attention of batches past 32 sequences, of a chunk among single rows on either path, and of
chunks of more units or sequences than the plan takes.  Tolerances as
tests/test_gpu_kv_attention.py derives them."""
import numpy as np
import pytest

from tests._step import starts
from tests.test_gpu_kv_nonfinite import Case

pytestmark = pytest.mark.gpu


def ragged(batch, cap, counts, seed):
    """Lengths from nothing to what the rows leave of cap."""
    rng = np.random.default_rng(seed)
    return [0 if rng.random() < 0.1 else int(rng.integers(0, cap - m + 1)) for m in counts]


@pytest.mark.parametrize("memory", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,dh,layout,batch,cap", [(8, 2, 64, "paged", 70, 640), (4, 4, 128, "slot", 33, 256),
                                                        (7, 1, 64, "head", 129, 128)])
def test_single_rows_of_many_sequences(hq, hkv, dh, layout, batch, cap, dtype, memory):
    counts = [int(i % 5 != 3) for i in range(batch)]
    c = Case(hq, hkv, dh, layout, cap, ragged(batch, cap, counts, batch), starts(counts).tolist(), 1, dtype)
    c.check(*c.run(memory))


@pytest.mark.parametrize("memory", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("batch", [3, 12, 45])
def test_a_chunk_among_single_rows(batch, dtype, memory):
    """500 rows of one sequence and a row or none of the others."""
    counts = [int(i % 4 > 0) for i in range(batch)]
    counts[batch // 2] = 500
    c = Case(8, 2, 64, "paged", 1024, ragged(batch, 1024, counts, batch), starts(counts).tolist(), 500, dtype)
    c.check(*c.run(memory))


@pytest.mark.parametrize("memory", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,batch,cap,most", [(2, 2, 260, 128, 104), (64, 8, 4, 1280, 1200)])
def test_chunks_without_a_plan(hq, hkv, batch, cap, most, dtype, memory):
    """More sequences than the plan takes, and more units."""
    counts = [most - i % 7 for i in range(batch)]
    c = Case(hq, hkv, 64, "slot", cap, ragged(batch, cap, counts, batch), starts(counts).tolist(), most, dtype)
    c.check(*c.run(memory))
