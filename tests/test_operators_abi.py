"""Argument checks of the entry points around the quantised layers, and the host functions among them: nothing here needs a GPU."""
import math

import numpy as np
import pytest

P = 0x10000  # a fake, 16-byte aligned, never dereferenced "device pointer"


@pytest.fixture(scope="module")
def B():
    from paper_2311_01305_amd import binding
    binding.load_library()
    return binding


def _refused(fn, ok, **changed):
    from paper_2311_01305_amd.binding import AweqError
    with pytest.raises(AweqError) as e:
        fn(**{**ok, **changed})
    return e.value.name


def test_quant_tokens(B):
    ok = dict(X=P, dt=B.AWEQ_F16, T=4, K=64, ldx=64, inv_s=P, xq=P, step_x=P, zero_x=P, rowsum_x=P, stream=0)
    bad = lambda **k: _refused(B.aweq_quant_tokens, ok, **k)
    for name in ("X", "xq", "step_x", "zero_x", "rowsum_x"):
        assert bad(**{name: None}) == "AWEQ_ERR_NULL"
    assert bad(dt=B.AWEQ_I8) == "AWEQ_ERR_DTYPE"
    assert bad(T=0) == bad(K=60, ldx=60) == bad(ldx=56) == bad(K=32776, ldx=32776) == "AWEQ_ERR_SHAPE"
    assert bad(X=P + 2) == bad(ldx=68) == bad(inv_s=P + 4) == bad(xq=P + 8) == "AWEQ_ERR_ALIGN"


def test_gemm_tokens(B):
    ok = dict(X=P, x_dt=B.AWEQ_BF16, T=4, K=64, ldx=64, inv_s=None, xq=P, step_x=P, zero_x=P, rowsum_x=P, wq=P, N=8, step_w=P, zero_w=P, w_group=0,
              rowsum_w=P, bias=P, out=P, out_dt=B.AWEQ_BF16, ldo=8, stream=0)
    bad = lambda **k: _refused(B.aweq_w8a8_gemm_tokens, ok, **k)
    for name in ("X", "xq", "step_x", "zero_x", "rowsum_x", "wq", "step_w", "zero_w", "rowsum_w", "out"):
        assert bad(**{name: None}) == "AWEQ_ERR_NULL"
    assert bad(w_group=128) == "AWEQ_ERR_GROUP"
    assert bad(out_dt=B.AWEQ_I8) == "AWEQ_ERR_DTYPE"
    assert bad(x_dt=7) == "AWEQ_ERR_DTYPE"
    assert bad(N=6) == bad(N=0) == bad(ldo=4) == bad(ldo=10) == bad(K=32776, ldx=32776) == bad(x_dt=B.AWEQ_I8, ldx=128) == "AWEQ_ERR_SHAPE"
    assert bad(out=P + 4) == bad(bias=P + 4) == bad(wq=P + 4) == bad(zero_w=P + 4) == bad(x_dt=B.AWEQ_I8, X=P + 8) == "AWEQ_ERR_ALIGN"


def test_rope_frequencies(B):
    f = np.zeros(64)
    B.aweq_rope_frequencies(128, 10000.0, f)
    want = np.array([10000.0 ** (-2 * i / 128) for i in range(64)])
    assert np.allclose(f, want, rtol=1e-14, atol=0)
    g = np.zeros(64)
    B.aweq_rope_frequencies(128, 10000.0, g, B.ROPE_LINEAR, 4.0)
    assert np.allclose(g, want / 4, rtol=1e-14, atol=0)
    B.aweq_rope_frequencies(128, 10000.0, g, B.ROPE_BASE, 4.0)
    assert g[0] == 1.0 and math.isclose(g[63], want[63] / 4, rel_tol=1e-12)
    B.aweq_rope_frequencies(128, 10000.0, g, B.ROPE_PARTS, 8.0, 8192.0, 1.0, 4.0)
    turns = 8192 * want / (2 * math.pi)
    kept = np.clip((turns - 1) / 3, 0, 1)
    assert np.allclose(g, kept * want + (1 - kept) * want / 8, rtol=1e-13, atol=0)
    assert (g[turns >= 4] == f[turns >= 4]).all() and np.allclose(g[turns <= 1], f[turns <= 1] / 8, rtol=1e-15)
    ok = dict(rot=128, base=10000.0, freq=g)
    bad = lambda **k: _refused(B.aweq_rope_frequencies, ok, **k)
    assert bad(freq=None) == "AWEQ_ERR_NULL"
    assert bad(rot=0) == bad(rot=7) == bad(base=0.0) == bad(base=math.inf) == bad(factor=0.0) == bad(factor=math.nan) == bad(kind=4) == bad(kind=-1) == "AWEQ_ERR_SHAPE"
    assert bad(rot=2, kind=B.ROPE_BASE) == bad(kind=B.ROPE_PARTS) == bad(kind=B.ROPE_PARTS, trained=10.0, low=4.0, high=4.0) == "AWEQ_ERR_SHAPE"


HEADS = dict(dt=1, T=3, Hq=8, Hk=2, D=128, ldq=1024, ldk=256, pos=P, freq=P, rot=128, interleaved=0, gain=1.0, q_norm=P, k_norm=P, eps=1e-5, q_out=P,
             ldqo=1024, stream=0)


def _heads(bad):
    assert bad(pos=None) == bad(freq=None) == bad(q_out=None) == bad(q=None) == "AWEQ_ERR_NULL"
    assert bad(dt=2) == "AWEQ_ERR_DTYPE"
    assert bad(T=0) == bad(D=0) == bad(D=264, ldq=4096, ldk=4096, ldqo=4096) == bad(D=100) == bad(Hq=0) == bad(Hk=-1) == "AWEQ_ERR_SHAPE"
    assert bad(rot=8) == bad(rot=136) == bad(rot=-16) == bad(rot=12, interleaved=1) == "AWEQ_ERR_SHAPE"
    assert bad(ldq=1016) == bad(ldk=248) == bad(ldqo=1016) == "AWEQ_ERR_SHAPE"
    assert bad(q=P + 2) == bad(k=P + 8) == bad(ldq=1028) == bad(ldk=260) == bad(ldqo=1028) == bad(q_out=P + 8) == bad(q_norm=P + 4) == bad(k_norm=P + 8) == "AWEQ_ERR_ALIGN"
    assert bad(pos=P + 2) == bad(freq=P + 4) == "AWEQ_ERR_ALIGN"


def test_qk_rope(B):
    ok = dict(HEADS, q=P, k=P, k_out=P, ldko=256)
    bad = lambda **k: _refused(B.aweq_qk_rope, ok, **k)
    _heads(bad)
    assert bad(q=None, k=None, q_out=None, k_out=None) == bad(k=None) == bad(k_out=None) == "AWEQ_ERR_NULL"
    assert bad(ldko=248) == "AWEQ_ERR_SHAPE"
    assert bad(k_out=P + 4) == bad(ldko=260) == "AWEQ_ERR_ALIGN"


def test_kv_append(B):
    ok = dict(HEADS, q=P, k=P, v=P, ldv=256, k_cache=P, v_cache=P, k_step=None, v_step=None, cache_dt=B.AWEQ_F16, pages=4, page_size=16, slot=P)
    bad = lambda **k: _refused(B.aweq_kv_append, ok, **k)
    _heads(bad)
    for name in ("k", "v", "k_cache", "v_cache", "slot"):
        assert bad(**{name: None}) == "AWEQ_ERR_NULL"
    assert bad(cache_dt=B.AWEQ_I8) == bad(cache_dt=B.AWEQ_I8, k_step=P) == "AWEQ_ERR_NULL"
    assert bad(cache_dt=B.AWEQ_BF16) == bad(dt=B.AWEQ_F32) == "AWEQ_ERR_DTYPE"
    assert bad(pages=0) == bad(page_size=8) == bad(page_size=512) == bad(page_size=48) == bad(ldv=248) == "AWEQ_ERR_SHAPE"
    assert bad(v=P + 8) == bad(ldv=260) == bad(k_cache=P + 8) == bad(slot=P + 4) == bad(cache_dt=B.AWEQ_I8, k_step=P + 4, v_step=P) == "AWEQ_ERR_ALIGN"


def test_prefix_attention(B):
    ok = dict(q=P, dt=B.AWEQ_F16, T=6, Hq=8, D=128, ldq=1024, k_cache=P, v_cache=P, k_step=None, v_step=None, cache_dt=B.AWEQ_F16, pages=64, page_size=16, Hk=2,
              prefix_table=P, prefix_len=100, table=P, table_ld=8, lens=P, q_start=P, B=3, max_len=128, max_q=4, scale=0.1, out=P, ldo=1024, lse=None, ws=P,
              ws_bytes=1 << 30, stream=0)
    bad = lambda **k: _refused(B.aweq_prefix_attention, ok, **k)
    for name in ("q", "k_cache", "v_cache", "prefix_table", "table", "lens", "out"):
        assert bad(**{name: None}) == "AWEQ_ERR_NULL"
    assert bad(cache_dt=B.AWEQ_I8) == "AWEQ_ERR_NULL"
    assert bad(dt=B.AWEQ_F32) == bad(cache_dt=B.AWEQ_BF16) == "AWEQ_ERR_DTYPE"
    assert bad(T=0) == bad(B=0) == bad(D=96) == bad(Hk=3) == bad(Hk=0) == bad(prefix_len=-1) == bad(max_len=-1) == bad(max_q=0) == bad(pages=0) == "AWEQ_ERR_SHAPE"
    assert bad(page_size=24) == bad(page_size=8) == bad(ldq=1016) == bad(ldo=1016) == bad(table_ld=0) == bad(q_start=None) == "AWEQ_ERR_SHAPE"
    assert bad(q=P + 8) == bad(out=P + 8) == bad(ldq=1028) == bad(ldo=1028) == bad(v_cache=P + 8) == bad(ws=P + 8) == "AWEQ_ERR_ALIGN"
    need = B.aweq_prefix_attention_ws(6, 8, 2, 128, 3, 4, 100, 128)
    assert need > 0
    assert bad(ws=None) == bad(ws_bytes=need - 1) == "AWEQ_ERR_WORKSPACE"
    # nothing to join, nothing to keep; what is no shape needs nothing either
    assert B.aweq_prefix_attention_ws(512, 64, 64, 128, 512, 1, 0, 128) == 0
    assert B.aweq_prefix_attention_ws(0, 8, 2, 128, 3, 4, 100, 128) == 0
