"""cc_kv_join where a part's weight is nothing in fp32: what the part holds does not matter, as
where it saw no slot; the largest part alone is the result, rounded as it was."""
import pytest
import torch

from tests._step import shape
from tests.test_gpu_kv_join import pkg  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("parts", [2, 3, 7])
def test_weights_that_vanish(pkg, parts, dtype):  # noqa: F811
    from paper_2607_27600_gb300 import cc
    n, hq, dh = 50, 4, 64
    g = torch.Generator(device="cuda").manual_seed(parts)
    x = [torch.full((n, hq, dh), float("nan"), dtype=dtype, device="cuda") for _ in range(parts)]
    lse = [torch.full((n, hq), -110.0 - 1e30 * (i % 2), device="cuda") for i in range(parts)]
    x[1], lse[1] = torch.randn(n, hq, dh, generator=g, device="cuda").to(dtype), torch.zeros(n, hq, device="cuda")
    out, joint = torch.empty_like(x[0]), torch.empty_like(lse[0])
    cc.cc_kv_join(shape(hq, 2, dh), x, lse, out, joint)
    assert torch.equal(out, x[1]) and torch.equal(joint, lse[1])   # (a weight and a sum of 1, exactly)
