"""cc_kv_compact of the longest sequence that it takes, exactly: counts and places whose
next steps pass 31 bits (layers without K and V: tokens, positions and totals alone)."""
import pytest
import torch

from tests._step import shape

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    import paper_2607_27600_gb300 as p
    p.load_library()
    return p


def test_a_sequence_next_to_31_bits(pkg):
    """All slots but one kept: those behind it move down by one."""
    from paper_2607_27600_gb300 import cc
    cap, gone = 2 ** 31 - 4224, 1000
    s = shape(8, 2, 64)
    tokens = torch.arange(cap, dtype=torch.int32, device="cuda")
    d = {"k": [None], "v": [None], "k_exp": [None], "v_exp": [None], "kv_block": 16, "tokens": tokens[None],
         "pos": (tokens ^ 5)[None], "seq_len": torch.tensor([cap], dtype=torch.int32, device="cuda")}
    cache = pkg.Cache(d)
    idx = torch.arange(cap, dtype=torch.int32, device="cuda")[None]
    idx[0, gone:] += 1
    count = torch.tensor([cap - 1], dtype=torch.int32, device="cuda")
    ws = cc.alloc_workspace(cc.cc_kv_compact_workspace_size(s, cache))
    cc.cc_kv_compact(s, cache, idx, count, ws)
    assert cc.cc_get_status() == cc.CC_OK
    kept = idx[0, :-1]
    assert torch.equal(d["tokens"][0, :-1], kept)
    assert torch.equal(d["pos"][0, :-1], kept ^ 5)
    assert d["seq_len"].tolist() == [cap - 1]
