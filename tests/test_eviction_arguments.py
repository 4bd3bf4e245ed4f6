"""What cc_kv_accumulate, cc_kv_compact and cc_kv_join refuse on the host, before
anything reaches a device (no GPU)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from tests.test_step_arguments import BASE, cache, cfg, lib, rows  # noqa: E402,F401


def accumulate(lib, c=None, kv=None, layer=0, r=None, dtype=0, first=0, memory=0, q=BASE, q_ld=512, lse=BASE,
               ws=BASE, ws_bytes=1 << 40):
    return lib.cc_kv_accumulate(c or cfg(), kv or cache(h2o_acc=BASE), layer, r or rows(), dtype, first, memory, q,
                                q_ld, lse, ws, ws_bytes, None)


def compact(lib, c=None, kv=None, idx=BASE, count=BASE, ws=BASE, ws_bytes=1 << 40):
    return lib.cc_kv_compact(c or cfg(), kv or cache(), idx, count, ws, ws_bytes, None)


def join(lib, c=None, dtype=0, n=4, k=2, part=(BASE, BASE), ld=(512, 512), lses=(BASE, BASE), out=BASE, out_ld=512):
    many = max(k, 1)
    ptrs = (ctypes.c_void_p * many)(*(list(part) * many)[:many])
    lds = (ctypes.c_int64 * many)(*(list(ld) * many)[:many])
    s = (ctypes.c_void_p * many)(*(list(lses) * many)[:many])
    return lib.cc_kv_join(c or cfg(), dtype, n, k, ptrs, lds, s, out, out_ld, None, None)


def test_nothing_to_do(lib):  # noqa: F811
    from paper_2607_27600_gb300 import cc
    none = rows(0, 0, None)
    assert accumulate(lib, r=none) == cc.CC_OK
    assert lib.cc_kv_accumulate_workspace_size(cfg(), cache(), none) == 0
    assert join(lib, n=0) == cc.CC_OK


def test_accumulate_is_checked(lib):  # noqa: F811
    from paper_2607_27600_gb300 import cc
    bad, none = cc.CC_ERR_INVALID_ARG, cc.CC_ERR_UNSUPPORTED
    for kw in (dict(kv=cache()), dict(first=1, memory=1), dict(q=None), dict(q=BASE + 8), dict(q_ld=511),
               dict(q_ld=516), dict(lse=None), dict(dtype=5), dict(dtype=-1), dict(layer=2), dict(layer=-1),
               dict(r=rows(4, 5)), dict(r=rows(4, 4, None)), dict(kv=cache(h2o_acc=BASE, kv_block=48)),
               dict(kv=cache(h2o_acc=BASE, seq_len=None))):
        assert accumulate(lib, **kw) == bad, kw
    for kw in (dict(dtype=2), dict(kv=cache(h2o_acc=BASE, kv_format=cc.KV_BF16)), dict(c=cfg(head_dim=96)),
               dict(kv=cache(h2o_acc=BASE, batch=1 << 16, cap=1 << 15))):
        assert accumulate(lib, **kw) == none, kw
    for r in (rows(), rows(200, 150)):
        need = lib.cc_kv_accumulate_workspace_size(cfg(), cache(), r)
        assert need > 0
        assert accumulate(lib, r=r, ws_bytes=need - 1) == cc.CC_ERR_WORKSPACE
        assert accumulate(lib, r=r, ws=None) == cc.CC_ERR_WORKSPACE
        assert accumulate(lib, r=r, ws=BASE + 8) == cc.CC_ERR_WORKSPACE


def test_compact_is_checked(lib):  # noqa: F811
    from paper_2607_27600_gb300 import cc
    bad, none = cc.CC_ERR_INVALID_ARG, cc.CC_ERR_UNSUPPORTED
    null, odd = (ctypes.c_void_p * 2)(None, None), (ctypes.c_void_p * 2)(BASE + 8, BASE)
    for kw in (dict(idx=None), dict(count=None), dict(kv=cache(tokens=None)), dict(kv=cache(pos=None)),
               dict(kv=cache(seq_len=None)), dict(kv=cache(k=odd)), dict(kv=cache(k_exp=null)),
               dict(kv=cache(kv_block=24)), dict(kv=cache(cap=200)), dict(kv=cache(batch=0)),
               dict(kv=cache(h_last=BASE + 2)), dict(kv=cache(block_table=BASE, page_size=64, n_pages=4)),
               dict(kv=cache(block_table=BASE, page_size=128, n_pages=4, kv_layout=1)), dict(kv=cache(kv_layout=2))):
        assert compact(lib, **kw) == bad, kw
        if "kv" in kw:
            assert lib.cc_kv_compact_workspace_size(cfg(), kw["kv"]) == 0
    for kw in (dict(kv=cache(kv_format=cc.KV_BF16)), dict(kv=cache(batch=1 << 16, cap=1 << 15)),
               dict(kv=cache(batch=65535, cap=128)), dict(c=cfg(head_dim=96))):
        assert compact(lib, **kw) == none, kw
    need = lib.cc_kv_compact_workspace_size(cfg(), cache())
    assert need > 0
    assert compact(lib, ws_bytes=need - 1) == cc.CC_ERR_WORKSPACE
    assert compact(lib, ws=None) == cc.CC_ERR_WORKSPACE
    # more arrays, more units; a layer without K and V has none
    long = cache(cap=1 << 16)
    need = lib.cc_kv_compact_workspace_size(cfg(), long)
    assert lib.cc_kv_compact_workspace_size(cfg(), cache(cap=1 << 16, h_last=BASE)) > need
    assert lib.cc_kv_compact_workspace_size(cfg(), cache(cap=1 << 16, k=null, v=null)) < need


def test_join_is_checked(lib):  # noqa: F811
    from paper_2607_27600_gb300 import cc
    bad = cc.CC_ERR_INVALID_ARG
    for kw in (dict(n=-1), dict(k=0), dict(dtype=3), dict(part=(BASE, None)), dict(part=(BASE + 8, BASE)),
               dict(ld=(512, 504)), dict(ld=(516, 512)), dict(lses=(None, BASE)), dict(out=None), dict(out=BASE + 4),
               dict(out_ld=500), dict(dtype=2, ld=(514, 512)), dict(ld=(512, 520))):
        assert join(lib, **kw) == bad, kw
    assert lib.cc_kv_join(cfg(), 0, 4, 2, None, None, None, BASE, 512, None, None) == bad
    assert join(lib, k=17) == cc.CC_ERR_UNSUPPORTED
    assert join(lib, c=cfg(head_dim=96)) == cc.CC_ERR_UNSUPPORTED
    wide = cfg(n_q_heads=32, n_kv_heads=8)
    assert join(lib, c=wide, n=(1 << 31) - 1, ld=(2048, 2048), out_ld=2048) == cc.CC_ERR_UNSUPPORTED


def test_binding_refuses_before_the_call():
    from paper_2607_27600_gb300 import cc
    x = torch.zeros(4, 8, 64)
    with pytest.raises(ValueError):
        cc.cc_kv_join(cfg(), [], [], x)
    with pytest.raises(ValueError):
        cc.cc_kv_join(cfg(), [x, x], [torch.zeros(4, 8)], x)
    with pytest.raises(TypeError):
        cc.cc_kv_join(cfg(), [x, None], [torch.zeros(4, 8)] * 2, x)
    with pytest.raises(TypeError):
        cc.cc_kv_join(cfg(), [x], [torch.zeros(4, 8)], x)   # not on a device


def test_sequences_next_to_31_bits(lib):  # noqa: F811
    from paper_2607_27600_gb300 import cc
    cap = (1 << 31) - 128
    assert accumulate(lib, kv=cache(h2o_acc=BASE, cap=cap, batch=1)) == cc.CC_ERR_UNSUPPORTED
    assert compact(lib, kv=cache(cap=cap, batch=1)) == cc.CC_ERR_UNSUPPORTED
