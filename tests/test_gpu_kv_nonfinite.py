"""cc_kv_attention of chunks whose keys, values, queries or pages are no numbers: a row with
a NaN or infinite score is 0, in units that are whole and in units that the plan cuts,
and the other rows are right.  Against the formula in 64 bits on the device;
tolerances as tests/test_gpu_kv_attention.py derives them."""
import numpy as np
import pytest
import torch

from tests._step import DeviceCache, columns, quantised, shape, starts, values

pytestmark = pytest.mark.gpu
TYPES = {"bf16": (torch.bfloat16, 2.0 ** -8), "f16": (torch.float16, 2.0 ** -11)}


def formula(q, k, v, lens, start, ok, memory):
    """Output, lse and sum_j p_j |V_j| of the rows (fp64, on the device): 0 and NaN for a row with
    a score that is no finite number; NaN where a row sees a value that is none."""
    group = q.shape[1] // k.shape[2]
    out, spread = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full(q.shape[:2], -torch.inf).to(q)
    for b, n in enumerate(lens):
        at, m = start[b], start[b + 1] - start[b]
        end = n if memory else n + m
        for h in range(q.shape[1] if ok[b] and m and end else 0):
            kk, vv = k[b, :end, h // group], v[b, :end, h // group]
            sees = torch.ones(m, end, dtype=torch.bool, device=q.device)
            if not memory:
                sees = torch.arange(end, device=q.device)[None] <= n + torch.arange(m, device=q.device)[:, None]
            x = q[at:at + m, h] @ kk.T / q.shape[2] ** 0.5
            none = (~x.isfinite() & sees).any(1, keepdim=True)
            p = torch.softmax(torch.where(none, 0.0, x).masked_fill(~sees, -torch.inf), 1)
            w = torch.nan_to_num(vv, nan=0.0)
            o = (p @ w).masked_fill((sees.double() @ vv.isnan().double()) > 0, torch.nan)
            out[at:at + m, h] = torch.where(none, 0.0, o)
            spread[at:at + m, h] = p @ w.abs()
            lse[at:at + m, h] = torch.where(none[:, 0], torch.nan,
                                            torch.logsumexp(x.masked_fill(~sees, -torch.inf), 1))
    return out, lse, spread


class Case:
    """A block-format cache, and rows [start[b], start[b + 1]) of each sequence."""

    def __init__(self, hq, hkv, dh, layout, cap, lens, start, most, dtype, seed=0):
        rng = np.random.default_rng(seed + cap)
        self.s, self.lens, self.start, self.most, self.layout = shape(hq, hkv, dh), lens, start, most, layout
        self.codes, self.exps = {}, {}
        for x in "kv":
            self.codes[x], self.exps[x] = quantised(rng, len(lens), cap, hkv, dh, 32)
        self.dtype, self.eps = TYPES[dtype]
        self.q = torch.from_numpy(rng.standard_normal((max(start), hq, dh)) * 1.5).to(self.dtype).double().numpy()

    def held(self, x):
        """Values of the cache's keys or values: an exponent of 0 is a scale of 0, 255 no number."""
        e = np.repeat(self.exps[x], 32, 1)[..., None]
        y = values(self.codes[x], self.exps[x])
        return np.where(e == 255, np.nan, np.where(e == 0, y * 0.0, y))

    def run(self, memory=False, lse=True, ok=None, status=0, pages=()):
        """The call's output and lse, and the formula's; pages: block-table entries
        (sequence, page) that lie outside the pool."""
        import paper_2607_27600_gb300 as pkg
        from paper_2607_27600_gb300 import cc
        c = DeviceCache(pkg, self.codes, self.exps, self.lens, self.layout)
        for b, page in pages:
            c.d["block_table"][b, page] = -3
        dq, = columns([self.q], self.dtype)
        n = len(dq)
        rows = pkg.Rows(n, torch.tensor(self.start, dtype=torch.int32, device="cuda"), None, self.most)
        ws = cc.alloc_workspace(cc.cc_kv_attention_workspace_size(self.s, c.cache, rows))
        ws.fill_(0xFF)
        out = torch.full(dq.shape, 7.0, dtype=self.dtype, device="cuda")
        ls = torch.full(dq.shape[:2], 7.0, device="cuda") if lse else None
        cc.cc_kv_attention(self.s, c.cache, 0, rows, dq, out, ws, lse=ls, memory_only=memory)
        assert cc.cc_get_status() == status
        k, v = (torch.from_numpy(self.held(x)).cuda() for x in "kv")
        want = formula(dq.double(), k, v, self.lens, self.start, ok or [True] * len(self.lens), memory)
        return out.double(), None if ls is None else ls.double(), want

    def check(self, got, ls, want, rows=slice(None)):
        got, (w, wl, spread) = got[rows], [x[rows] for x in want]
        assert torch.equal(got.isnan(), w.isnan())
        p = 2.0 ** (-8 if self.dtype is torch.bfloat16 else -11)
        f = ~w.isnan()
        assert ((got - w).abs() <= self.eps * w.abs() + 2 * p * spread + 1e-30)[f].all()
        zero = wl.isnan()   # a score that is no number
        assert (got[zero] == 0).all()
        if ls is not None:
            ls = ls[rows]
            assert not ls[zero].isfinite().any()
            assert torch.equal(ls[wl.isinf()], wl[wl.isinf()])   # rows that see no slot
            f = wl.isfinite()
            assert ((ls - wl).abs()[f] <= 2.0 ** -12 + 2.0 ** -22 * wl[f].abs()).all()


# whole units, and few long ones that the plan cuts
SIZES = {"whole": (8, 2, 64, "paged", 512, [300, 3], [0, 100, 250], 150),
         "cut": (8, 2, 128, "paged", 8192, [8000], [0, 120], 120)}


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("size", list(SIZES))
@pytest.mark.parametrize("memory", [False, True])
def test_rows_with_a_score_that_is_no_number(size, dtype, memory):
    """A NaN code in a key of the memory, which every row sees, and in a new token's, which the
    later rows do; infinite and NaN queries."""
    c = Case(*SIZES[size], dtype)
    n, m = c.lens[0], c.start[1]
    c.codes["k"][0, n // 2, 1, 9] = 0x7F
    c.codes["k"][0, n + m // 2, 0, 5] = 0xFF
    c.q[3, 0, 7], c.q[4, 1, 7], c.q[m - 1, 2, 0] = np.inf, -np.inf, np.nan
    got, ls, want = c.run(memory)
    assert want[1][:m, 4:].isnan().all() and want[1][0, :4].isfinite().all()
    assert want[1][m // 2:m, :4].isnan().all() == (not memory)
    c.check(got, ls, want)
    again = c.run(memory, lse=False)[0]
    assert torch.equal(again.isnan(), got.isnan()) and torch.equal(again.nan_to_num(), got.nan_to_num())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("size", list(SIZES))
def test_rows_that_see_a_bad_page(size, dtype):
    """A block-table entry outside the pool is reported; the rows that would see its slots are 0, the
    other sequences right."""
    from paper_2607_27600_gb300 import cc
    c = Case(*SIZES[size], dtype)
    got, _, want = c.run(status=cc.CC_ERR_DEVICE_ARG, pages=[(0, 1)])
    assert (got[:c.start[1]] == 0).all()
    c.check(got, None, want, slice(c.start[1], None))


@pytest.mark.parametrize("lse", [True, False])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("size", list(SIZES))
def test_a_token_that_is_no_number(size, dtype, lse):
    """A new token whose keys, values and query are all NaN, as a diverged one's are: its own and
    the later rows are 0, not NaN; a NaN among the values alone is NaN in its column."""
    c = Case(*SIZES[size], dtype)
    n, m = c.lens[0], c.start[1]
    for x in "kv":
        c.codes[x][0, n + m - 30] = 0x7F
    c.q[m - 30] = np.nan
    c.codes["v"][0, n + 11, 1, 6] = 0xFF
    got, ls, want = c.run(lse=lse)
    assert want[0][11:m - 30, 4:, 6].isnan().all() and (want[0][m - 30:m] == 0).all()
    c.check(got, ls, want)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_not_a_number_beside_rows_out_of_order(dtype):
    """Bad sequences (too many rows, and an end before the start) are reported; a NaN value of a
    good one, whose rows lie before the end of a bad one's, is still NaN in its column."""
    from paper_2607_27600_gb300 import cc
    c = Case(8, 2, 64, "slot", 512, [100, 100, 100], [0, 290, 150, 300], 150, dtype)
    c.codes["v"][2, 100 + 40, 0, 21] = 0x7F
    got, ls, want = c.run(ok=[False, False, True], status=cc.CC_ERR_DEVICE_ARG)
    assert want[0][190:, :4, 21].isnan().all()
    c.check(got, ls, want, slice(150, 300))
