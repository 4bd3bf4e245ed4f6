"""cc_kv_accumulate of single rows over caches with room for many slots, whose steps take three
CTAs an SM: ragged sequences, head groups, types and dims; against the fp64 oracle, with the
tolerances of test_gpu_kv_accumulate.py."""
import numpy as np
import pytest
import torch

from tests._step import columns, device_rows
from tests.test_gpu_kv_accumulate import Case, pkg  # noqa: F401

pytestmark = pytest.mark.gpu

CASES = [
    # hq, hkv, dh, block, layout, dtype, cap, lens, counts: batch * cap / 16 steps > 3 * 128 an SM
    (8, 2, 64, 64, "slot", "bf16", 32768, 32, 1),
    (4, 1, 64, 16, "paged", "f16", 65536, 16, 1),
    (7, 1, 128, 128, "head", "bf16", 65536, 15, 1),
    (4, 2, 128, 32, "slot", "f16", 32768, 30, 1),
    (2, 1, 64, 64, "paged", "bf16", 65536, 16, 4),   # four rows of two heads: one eight of rows
]


class Roomy(Case):
    """A case in buffers of `room` slots a sequence, of which only the first ones are ever held."""

    def widen(self, room):
        d, cap = self.c.d, self.c.cap
        b, extra = len(self.lens), room - cap
        for n in ("k", "k_exp"):   # (the values take no part)
            d[n] = d[n.replace("k", "v", 1)] = [grow(self.c, d[n][0], extra if n == "k" else extra // self.c.block)]
        for n in ("tokens", "pos"):
            d[n] = torch.zeros(b, room, dtype=torch.int32, device="cuda")
        if "block_table" in d:   # (the others are no pages)
            more = torch.full((b, extra // self.c.page), -7, dtype=torch.int32, device="cuda")
            d["block_table"] = torch.cat([d["block_table"], more], 1).contiguous()
        self.room = room

    def run(self, first=False):
        from paper_2607_27600_gb300 import cc
        dq, = columns([self.q], self.t, 24)
        cap = self.c.cap
        acc = torch.full((len(self.lens), self.room), 3.0, device="cuda")
        acc[:, :cap] = torch.from_numpy(self.acc).cuda()
        cache = self.pkg.Cache({**self.c.d, "h2o_acc": acc})
        rows = device_rows(self.pkg, self.counts)
        ws = cc.alloc_workspace(cc.cc_kv_accumulate_workspace_size(self.s, cache, rows))
        cc.cc_kv_accumulate(self.s, cache, 0, rows, dq, torch.from_numpy(self.lse).cuda(), ws, first=first,
                            memory_only=self.memory)
        assert (acc[:, cap:] == 3).all()
        return acc[:, :cap].cpu().numpy()


def grow(c, t, extra):
    """`extra` more places along a buffer's slots (a pool stays as it is)."""
    if c.layout == "paged":
        return t
    at = 2 if c.layout == "head" else 1
    pad = list(t.shape)
    pad[at] = extra
    return torch.cat([t, torch.full(pad, 0x7F, dtype=torch.uint8, device="cuda")], at).contiguous()


@pytest.mark.parametrize("memory", [False, True])
@pytest.mark.parametrize("hq,hkv,dh,block,layout,dtype,cap,batch,most", CASES)
def test_matches_oracle(pkg, hq, hkv, dh, block, layout, dtype, cap, batch, most, memory):  # noqa: F811
    from paper_2607_27600_gb300 import cc
    assert batch * cap // 16 > 3 * 128 * torch.cuda.get_device_properties(0).multi_processor_count
    rng = np.random.default_rng(cap + hq)
    lens = [int(x) for x in rng.integers(0, 3000, batch)]
    lens[0], lens[1], lens[2] = 0, 1, 6000
    counts = [1] * batch if most == 1 else [int(x) for x in rng.integers(0, most + 1, batch)]
    counts[3] = most
    c = Roomy(pkg, hq * 1000 + dh, hq, hkv, dh, block, layout, dtype, 6144, lens, counts, memory)
    c.widen(cap)
    for first in (False, not memory):
        got = c.run(first=first)
        assert cc.cc_get_status() == cc.CC_OK
        c.check(got, first=first)
        np.testing.assert_array_equal(c.run(first=first), got)
