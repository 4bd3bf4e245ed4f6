"""cc_kv_attention where scores are far larger than fp32 holds whole numbers for: the row is
the value of its largest key, whatever that value's scale; a single key is that key's value.
(The gap to the second key is checked to be far past the scores' rounding.)"""
import numpy as np
import pytest
import torch

import oracle
from tests._step import DeviceCache, columns, device_rows, quantised, shape, starts, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("power,dh,lens,counts", [
    (power, *case) for power in (14, 24, 27, 31, 36, 70)
    for case in ((64, [200, 0, 77], [1, 1, 1]), (128, [1, 500], [9, 2]), (64, [3000], [1]), (64, [100], [200]),
                 (64, [3000], [60])) if power < 36 or max(case[2]) < 60])   # (chunks reach to 2^30)
def test_large_scores(power, dh, lens, counts, dtype):
    import paper_2607_27600_gb300 as pkg
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(7)
    t, eps = (torch.bfloat16, 2.0 ** -8) if dtype == "bf16" else (torch.float16, 2.0 ** -11)
    s, b, cap, n = shape(4, 2, dh), len(lens), 3072 if max(lens) > 512 else 512, sum(counts)
    codes, exps = {}, {}
    for x in "kv":
        codes[x], exps[x] = quantised(rng, b, cap, 2, dh, 32)
    exps["v"] = (exps["v"].astype(int) + rng.integers(-6, 7, exps["v"].shape)).astype(np.uint8)
    # scores of up to about 2^power in size (fp16 queries are small: the keys make up for it)
    up = power - 4 if dtype == "bf16" else 10
    exps["k"] = (exps["k"].astype(int) + power - 4 - up).astype(np.uint8)
    q = torch.from_numpy(rng.standard_normal((n, 4, dh)) * 2.0 ** up).to(t).double().numpy()
    k, v = values(codes["k"], exps["k"]), values(codes["v"], exps["v"])
    want, want_lse, _ = oracle.attend_rows(q, k, v, lens, starts(counts))
    c = DeviceCache(pkg, codes, exps, lens, "slot")
    dq, = columns([q], t)
    rows = device_rows(pkg, counts)
    out, ls = torch.empty(n, 4, dh, dtype=t, device="cuda"), torch.empty(n, 4, device="cuda")
    ws = cc.alloc_workspace(cc.cc_kv_attention_workspace_size(s, c.cache, rows))
    cc.cc_kv_attention(s, c.cache, 0, rows, dq, out, ws, lse=ls)
    assert cc.cc_get_status() == cc.CC_OK
    got, ls = out.double().cpu().numpy(), ls.double().cpu().numpy()
    clear, st = np.zeros((n, 4), bool), starts(counts)
    for i in range(b):
        for r in range(st[i], st[i + 1]):
            for h in range(4):
                x = np.sort(k[i, :lens[i] + r - st[i] + 1, h // 2] @ q[r, h]) / np.sqrt(dh)
                # fp32 sums of dh terms: 2^-18 of the row's largest, with room
                clear[r, h] = len(x) == 1 or x[-1] - x[-2] > 40 + 2.0 ** -17 * np.abs(x).max()
    assert clear.mean() > 0.5
    # the output's rounding, and one of its key's probability (bf16 in a chunk)
    p = 2.0 ** (-8 if dtype == "bf16" and max(counts) > 32 else -11)
    assert (np.abs(got - want) <= (eps + 2 * p) * np.abs(want) + 1e-30)[clear].all()
    assert (np.abs(ls - want_lse) <= 1 + 2.0 ** -17 * np.abs(want_lse))[clear].all()


def test_scores_below_every_usual_one():
    """One key whose score is finite and below -2^100: its value, not an empty row."""
    import paper_2607_27600_gb300 as pkg
    from paper_2607_27600_gb300 import cc
    rng = np.random.default_rng(8)
    s, codes, exps = shape(4, 2, 64), {}, {}
    for x in "kv":
        codes[x], exps[x] = quantised(rng, 2, 128, 2, 64, 32)
    exps["k"] += 40
    c = DeviceCache(pkg, codes, exps, [0, 0], "slot")
    k, v = values(codes["k"], exps["k"]), values(codes["v"], exps["v"])
    q = np.repeat(-np.sign(k[:, 0]), 2, 1) * 2.0 ** 70
    dq, = columns([q], torch.bfloat16)
    out, ls = torch.empty(2, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 4, device="cuda")
    rows = pkg.Rows(2)
    ws = cc.alloc_workspace(cc.cc_kv_attention_workspace_size(s, c.cache, rows))
    cc.cc_kv_attention(s, c.cache, 0, rows, dq, out, ws, lse=ls)
    assert cc.cc_get_status() == cc.CC_OK
    want, want_lse, _ = oracle.attend_rows(q, k, v, [0, 0], [0, 1, 2])
    assert want_lse.max() < -1e30
    assert (np.abs(out.double().cpu().numpy() - want) <= (2.0 ** -8 + 2.0 ** -10) * np.abs(want)).all()
    assert (np.abs(ls.double().cpu().numpy() / want_lse - 1) < 2.0 ** -18).all()
