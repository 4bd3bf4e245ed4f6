"""cc_kv_advance reports a negative position, which it takes as 0."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_a_negative_position_is_reported():
    import paper_2607_27600_gb300 as pkg
    from paper_2607_27600_gb300 import cc
    z = lambda: torch.zeros(2, 64, 1, 64, dtype=torch.uint8, device="cuda")   # noqa: E731
    e = lambda: torch.zeros(2, 4, 1, dtype=torch.uint8, device="cuda")        # noqa: E731
    d = {"k": [z()], "v": [z()], "k_exp": [e()], "v_exp": [e()], "kv_block": 16,
         "seq_len": torch.tensor([3, 5], dtype=torch.int32, device="cuda"),
         "tokens": torch.zeros(2, 64, dtype=torch.int32, device="cuda"),
         "pos": torch.full((2, 64), 9, dtype=torch.int32, device="cuda")}
    cache = pkg.Cache(d)
    for pos, status in (([7, -1], cc.CC_ERR_DEVICE_ARG), ([8, 2], cc.CC_OK)):
        rows = pkg.Rows(2, pos=torch.tensor(pos, dtype=torch.int32, device="cuda"))
        cc.cc_kv_advance(cache, rows)
        assert cc.cc_get_status() == status
    assert d["seq_len"].tolist() == [5, 7]
    assert d["pos"][0, 3:5].tolist() == [7, 8] and d["pos"][1, 5:7].tolist() == [0, 2]
