"""What the serving step's calls refuse on the host, before anything reaches a device
(no GPU): the C ABI's checks, the binding's, and the calls that refuse the block
format."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

BASE = 1 << 20   # addresses only: none is dereferenced on these paths


@pytest.fixture(scope="module")
def lib():
    from paper_2607_27600_gb300 import build, cc
    build.build_library()
    return cc.load_library()


def cfg(**kw):
    from paper_2607_27600_gb300 import cc
    v = dict(n_layers=2, d_model=256, n_q_heads=8, n_kv_heads=2, head_dim=64, d_ff=384, vocab=1000,
             rope_theta=1e4, rms_eps=1e-5)
    v.update(kw)
    return cc.cc_model_cfg(*v.values())


def cache(**kw):
    from paper_2607_27600_gb300 import cc
    two = (ctypes.c_void_p * 2)(BASE, BASE)
    c = cc.cc_kv_cache()
    c.batch, c.cap, c.seq_len, c.k, c.v, c.tokens, c.pos = 2, 256, BASE, two, two, BASE, BASE
    c.kv_format, c.kv_block, c.k_exp, c.v_exp = cc.KV_E4M3_BLOCK, 32, two, two
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rows(n=4, most=4, start=BASE, pos=None):
    from paper_2607_27600_gb300 import cc
    return cc.cc_rows(n, most, start, pos)


def append(lib, c=None, kv=None, layer=0, r=None, dtype=0, k=BASE, k_ld=128, v=BASE, v_ld=128, q=None, q_ld=0,
           qo=None, qo_ld=0):
    return lib.cc_kv_append(c or cfg(), kv or cache(), layer, r or rows(), dtype, 1, k, k_ld, v, v_ld, q, q_ld,
                            qo, qo_ld, None)


def attend(lib, c=None, kv=None, layer=0, r=None, dtype=0, q=BASE, q_ld=512, out=BASE, out_ld=512, ws=BASE,
           ws_bytes=1 << 40):
    return lib.cc_kv_attention(c or cfg(), kv or cache(), layer, r or rows(), dtype, 0, q, q_ld, out, out_ld,
                               None, ws, ws_bytes, None)


def test_nothing_to_do(lib):
    from paper_2607_27600_gb300 import cc
    none = rows(0, 0, None)
    assert append(lib, r=none) == cc.CC_OK
    assert attend(lib, r=none) == cc.CC_OK
    assert lib.cc_kv_advance(cache(), none, None, None) == cc.CC_OK
    assert lib.cc_kv_attention_workspace_size(cfg(), cache(), none) == 0
    assert lib.cc_token_logprobs(BASE, 0, 0, 10, 10, None, None, None, 0, None, None, None) == cc.CC_OK


def test_structs_match_the_header():
    from paper_2607_27600_gb300 import cc
    from tests.test_abi import _header_struct_fields, header_enums
    assert [f[0] for f in cc.cc_rows._fields_] == _header_struct_fields("cc_rows")
    e = header_enums()
    assert e["CC_KV_E4M3_BLOCK"] == cc.KV_E4M3_BLOCK
    assert {torch.bfloat16: e["CC_BF16"], torch.float16: e["CC_F16"], torch.float32: e["CC_F32"]} == cc.DTYPES


def test_rows_and_cache_are_checked(lib):
    from paper_2607_27600_gb300 import cc
    bad, none = cc.CC_ERR_INVALID_ARG, cc.CC_ERR_UNSUPPORTED
    for call in (append, attend):
        for r in (rows(-1), rows(4, 0), rows(4, 5), rows(4, 4, None), rows(2, 2, None), rows(3, 1, None)):
            assert call(lib, r=r) == bad
        for layer in (-1, 2):
            assert call(lib, layer=layer) == bad
        null = (ctypes.c_void_p * 2)(None, BASE)
        odd = (ctypes.c_void_p * 2)(BASE + 8, BASE)
        for kv in (cache(batch=0), cache(cap=0), cache(seq_len=None), cache(k=null), cache(v=odd),
                   cache(k_exp=null), cache(v_exp=odd), cache(kv_block=8), cache(kv_block=48), cache(kv_block=256),
                   cache(cap=200), cache(kv_layout=2), cache(kv_format=7),
                   cache(block_table=BASE, page_size=64, n_pages=4), cache(block_table=BASE, page_size=128, n_pages=0),
                   cache(block_table=BASE, page_size=128, n_pages=4, kv_layout=1)):
            assert call(lib, kv=kv) == bad
        assert call(lib, kv=cache(batch=1 << 16, cap=1 << 15)) == none
        assert call(lib, c=cfg(head_dim=96)) == none
        assert call(lib, c=cfg(n_kv_heads=3)) == bad
    # any layer but the one that is asked for may be missing
    assert lib.cc_kv_advance(cache(pos=None), rows(), None, None) == bad
    assert lib.cc_kv_advance(cache(tokens=None), rows(), BASE, None) == bad


def test_buffers_are_checked(lib):
    from paper_2607_27600_gb300 import cc
    bad = cc.CC_ERR_INVALID_ARG
    for kw in (dict(k=None), dict(v=None), dict(k=BASE + 2), dict(k_ld=120), dict(v_ld=129), dict(v_ld=132),
               dict(q=BASE, q_ld=512), dict(qo=BASE, qo_ld=512), dict(q=BASE, q_ld=512, qo=BASE + 4, qo_ld=512),
               dict(q=BASE, q_ld=504, qo=BASE, qo_ld=512), dict(dtype=3), dict(dtype=-1), dict(dtype=2, k_ld=130)):
        assert append(lib, **kw) == bad, kw
    assert append(lib, kv=cache(pos=None)) == bad   # positions neither given nor in the cache
    for kw in (dict(q=None), dict(out=None), dict(q=BASE + 8), dict(q_ld=511), dict(out_ld=516), dict(dtype=5)):
        assert attend(lib, **kw) == bad, kw
    assert attend(lib, dtype=2) == cc.CC_ERR_UNSUPPORTED
    assert attend(lib, kv=cache(kv_format=cc.KV_BF16)) == cc.CC_ERR_UNSUPPORTED
    for r in (rows(), rows(200, 150)):   # the direct kernel's workspace and the tile attention's
        need = lib.cc_kv_attention_workspace_size(cfg(), cache(), r)
        assert need > 0
        assert attend(lib, r=r, ws_bytes=need - 1) == cc.CC_ERR_WORKSPACE
        assert attend(lib, r=r, ws=None) == cc.CC_ERR_WORKSPACE
    # the copy of the layer is part of the larger one
    assert lib.cc_kv_attention_workspace_size(cfg(), cache(), rows(200, 150)) >= 2 * 2 * 256 * 2 * 64 * 2


def test_logits_are_checked(lib):
    from paper_2607_27600_gb300 import cc

    def call(z=BASE, dtype=0, n=2, vocab=100, ld=100, t=None, lp=None, top=0, ids=None):
        return lib.cc_token_logprobs(z, dtype, n, vocab, ld, t, lp, None, top, ids, None, None)

    bad = cc.CC_ERR_INVALID_ARG
    for kw in (dict(z=None), dict(z=BASE + 1), dict(z=BASE + 2, dtype=2), dict(dtype=9), dict(n=-1), dict(vocab=0),
               dict(ld=99), dict(t=BASE), dict(lp=BASE), dict(top=-1), dict(top=101, ids=BASE)):
        assert call(**kw) == bad, kw
    assert call(top=33, ids=BASE) == cc.CC_ERR_UNSUPPORTED


def test_other_calls_refuse_the_block_format(lib):
    from paper_2607_27600_gb300 import cc
    none = cc.CC_ERR_UNSUPPORTED
    c, kv = cfg(), cache()
    w = cc.cc_model_weights(BASE, BASE, BASE, (cc.cc_layer_weights * 2)())
    kv.h_last = BASE
    assert lib.cc_score_layer(c, w, kv, 0, BASE, BASE, 1 << 40, None) == none
    assert lib.cc_score_full(c, w, kv, 0, BASE, BASE, 1 << 40, None) == none
    assert lib.cc_append_chunk(c, w, kv, BASE, None, BASE, 4, BASE, 1 << 40, None) == none
    assert lib.cc_decode_step(c, w, kv, BASE, BASE, None, BASE, 1 << 40, None) == none
    assert lib.cc_compact_kv(c, kv, BASE, BASE, BASE, 1 << 40, None) == none
    assert lib.cc_compact_workspace_size(c, kv) == 0
    assert lib.cc_score_importance(c, kv, BASE, BASE, 1 << 40, None) == none


def test_binding_refuses_before_the_call():
    from paper_2607_27600_gb300 import cc
    x = torch.zeros(4, 2, 64)
    with pytest.raises(TypeError):
        cc._row_ptr(x, "k", 4, 128, x.dtype)   # not on a device
    with pytest.raises(ValueError):
        cc.Rows(4, row_start=torch.zeros(3))
    with pytest.raises(ValueError):
        cc.Rows(4, pos=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        cc._vec_ptr(torch.zeros(3), "lse", 4, torch.float32)
    with pytest.raises(ValueError):
        cc._dtype(torch.zeros(1, dtype=torch.float64), "k")
    codes, exps = torch.zeros(1, 64, 2, 64, dtype=torch.uint8), torch.zeros(1, 2, 2, dtype=torch.uint8)
    cc.Cache._check_block({"k": [codes], "v": [None], "k_exp": [exps], "v_exp": [None]}, 32)
    for bad in (dict(k_exp=[exps[:, :1]]), dict(k_exp=[]), dict(k=[codes.half()]), dict(k_exp=[exps.int()])):
        with pytest.raises(ValueError):
            cc.Cache._check_block({**{"k": [codes], "v": [None], "k_exp": [exps], "v_exp": [None]}, **bad}, 32)
