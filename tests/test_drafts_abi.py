"""Argument checks of the entry points for 4-bit projections and drafted tokens, and their host functions: nothing here needs a GPU."""
import pytest

P = 0x10000  # a fake, 16-byte aligned, never dereferenced "device pointer"
Q = 0x90000000


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


def test_sizes(B):
    assert B.aweq_mx4_code_bytes(3, 32) == 3 * 64 and B.aweq_mx4_scale_bytes(3, 32) == 3 * 16
    assert B.aweq_mx4_code_bytes(5, 544) == 5 * 5 * 64 and B.aweq_mx4_scale_bytes(5, 544) == 5 * 2 * 16
    assert B.aweq_mx4_code_bytes(2 ** 31 - 1, 4096) == (2 ** 31 - 1) * 32 * 64
    for rows, K in ((0, 32), (1, 0), (1, 33), (1, 16), (2 ** 31, 32), (1, 2 ** 20 + 32), (-1, 32)):
        assert B.aweq_mx4_code_bytes(rows, K) == B.aweq_mx4_scale_bytes(rows, K) == 0


def test_quant_mx4(B):
    ok = dict(X=P, dt=B.AWEQ_F16, rows=4, K=64, ldx=64, factor=P, codes=P, scales=P, stream=0)
    bad = lambda **k: _refused(B.aweq_quant_mx4, ok, **k)
    for name in ("X", "codes", "scales"):
        assert bad(**{name: None}) == "AWEQ_ERR_NULL"
    assert bad(dt=B.AWEQ_I8) == bad(dt=9) == "AWEQ_ERR_DTYPE"
    assert bad(rows=0) == bad(rows=2 ** 31) == bad(K=48) == bad(K=0) == bad(ldx=56) == bad(K=2 ** 20 + 32, ldx=2 ** 21) == "AWEQ_ERR_SHAPE"
    assert bad(X=P + 2) == bad(ldx=68) == bad(factor=P + 4) == bad(codes=P + 8) == bad(scales=P + 4) == bad(dt=B.AWEQ_F32, ldx=66) == "AWEQ_ERR_ALIGN"


def test_mx4_values(B):
    ok = dict(codes=P, scales=P, rows=4, K=64, out=P, out_dt=B.AWEQ_BF16, ldo=64, stream=0)
    bad = lambda **k: _refused(B.aweq_mx4_values, ok, **k)
    for name in ("codes", "scales", "out"):
        assert bad(**{name: None}) == "AWEQ_ERR_NULL"
    assert bad(out_dt=B.AWEQ_I8) == "AWEQ_ERR_DTYPE"
    assert bad(rows=0) == bad(K=40) == bad(ldo=56) == "AWEQ_ERR_SHAPE"
    assert bad(out=P + 8) == bad(ldo=68) == bad(codes=P + 4) == bad(scales=P + 8) == "AWEQ_ERR_ALIGN"


def test_mx4_gemm_tokens(B):
    ok = dict(X=P, x_dt=B.AWEQ_BF16, T=4, K=64, ldx=64, factor=None, xq=P, x_scale=P, wq=P, w_scale=P, N=8, bias=P, out=P, out_dt=B.AWEQ_BF16, ldo=8, stream=0)
    bad = lambda **k: _refused(B.aweq_mx4_gemm_tokens, ok, **k)
    for name in ("xq", "x_scale", "wq", "w_scale", "out"):
        assert bad(**{name: None}) == "AWEQ_ERR_NULL"
    assert bad(out_dt=B.AWEQ_I8) == bad(x_dt=B.AWEQ_I8) == "AWEQ_ERR_DTYPE"
    for given in (False, True):
        more = dict(X=None) if given else {}
        assert bad(N=6, **more) == bad(N=0, **more) == bad(ldo=4, **more) == bad(ldo=10, **more) == bad(K=48, **more) == bad(T=0, **more) == "AWEQ_ERR_SHAPE"
        assert bad(T=2 ** 31, **more) == bad(N=2 ** 31, ldo=2 ** 31, **more) == "AWEQ_ERR_SHAPE"
        assert bad(out=P + 4, **more) == bad(bias=P + 4, **more) == bad(wq=P + 4, **more) == bad(w_scale=P + 8, **more) == bad(xq=P + 8, **more) == "AWEQ_ERR_ALIGN"
    assert bad(ldx=56) == "AWEQ_ERR_SHAPE" and bad(X=P + 8) == bad(ldx=68) == bad(factor=P + 4) == "AWEQ_ERR_ALIGN"


def test_step_plan(B):
    ok = dict(lens=P, change=P + 0x1000, B=3, page_size=16, pages=64, table=P + 0x2000, table_ld=8, table_pages=8, free_pages=P + 0x3000, free_count=P + 0x4000,
              prefix_len=0, T=9, lens_out=P + 0x5000, count_out=P + 0x6000, q_start=P + 0x7000, pos=P + 0x8000, slot=P + 0x9000, stream=0)
    bad = lambda **k: _refused(B.aweq_step_plan, ok, **k)
    for name in ("lens", "change", "table", "free_pages", "free_count", "lens_out", "count_out", "q_start", "pos", "slot"):
        assert bad(**{name: None}) == "AWEQ_ERR_NULL"
    assert bad(B=0) == bad(B=8193) == bad(T=0) == bad(T=2 ** 24 + 1) == bad(page_size=8) == bad(page_size=48) == bad(page_size=512) == bad(pages=0) == "AWEQ_ERR_SHAPE"
    assert bad(pages=2 ** 31) == bad(table_pages=0) == bad(table_pages=9) == bad(table_ld=7) == bad(prefix_len=-1) == bad(prefix_len=2 ** 29 + 1) == "AWEQ_ERR_SHAPE"
    assert bad(table_pages=2 ** 22, table_ld=2 ** 22, page_size=256, table=Q) == "AWEQ_ERR_SHAPE"
    assert bad(lens=P + 2) == bad(slot=P + 0x9004) == bad(pos=P + 0x8001) == "AWEQ_ERR_ALIGN"
    assert bad(lens_out=P) == bad(count_out=P + 0x4000) == bad(pos=P + 0x1000 - 4) == bad(q_start=P + 0x2000) == bad(slot=P + 0x3000) == "AWEQ_ERR_ALIGN"


def test_tree_mask(B):
    ok = dict(parent=P, T=9, q_start=P, B=3, max_q=70, lens=P, prefix_len=0, mask=P, mask_ld=2, pos=P, stream=0)
    bad = lambda **k: _refused(B.aweq_tree_mask, ok, **k)
    for name in ("parent", "q_start", "mask", "lens"):
        assert bad(**{name: None}) == "AWEQ_ERR_NULL"
    assert bad(T=0) == bad(T=2 ** 24 + 1) == bad(B=0) == bad(B=2 ** 20 + 1) == bad(max_q=0) == bad(max_q=4097, mask_ld=80) == bad(mask_ld=1) == bad(prefix_len=-1) == "AWEQ_ERR_SHAPE"
    assert bad(parent=P + 1) == bad(mask=P + 4) == bad(pos=P + 2) == bad(lens=P + 2) == "AWEQ_ERR_ALIGN"
    apart = dict(parent=P + 0x1000, q_start=P + 0x2000, lens=P + 0x3000, mask=P + 0x4000, pos=P + 0x5000)
    for name in ("parent", "q_start", "lens"):
        assert bad(**{**apart, "pos": apart[name] + 4}) == bad(**{**apart, "mask": apart[name] - 8}) == "AWEQ_ERR_ALIGN"


def test_tree_attention(B):
    ok = dict(q=P, dt=B.AWEQ_F16, T=6, Hq=8, D=128, ldq=1024, k_cache=P, v_cache=P, k_step=None, v_step=None, cache_dt=B.AWEQ_F16, pages=64, page_size=16, Hk=2,
              prefix_table=P, prefix_len=100, table=P, table_ld=8, lens=P, q_start=P, B=3, max_len=128, max_q=4, mask=P, mask_ld=1, scale=0.1, out=P, ldo=1024, lse=None,
              ws=P, ws_bytes=1 << 30, stream=0)
    bad = lambda **k: _refused(B.aweq_tree_attention, ok, **k)
    for name in ("q", "k_cache", "v_cache", "prefix_table", "table", "lens", "out", "mask", "q_start"):
        assert bad(**{name: None}) == "AWEQ_ERR_NULL"
    assert bad(cache_dt=B.AWEQ_I8) == "AWEQ_ERR_NULL"
    assert bad(dt=B.AWEQ_F32) == bad(cache_dt=B.AWEQ_BF16) == "AWEQ_ERR_DTYPE"
    assert bad(T=0) == bad(B=0) == bad(D=96) == bad(Hk=3) == bad(prefix_len=-1) == bad(max_q=0) == bad(pages=0) == bad(mask_ld=0) == bad(scale=0.0) == "AWEQ_ERR_SHAPE"
    assert bad(T=200, max_q=65) == bad(page_size=24) == bad(ldq=1016) == bad(ldo=1016) == bad(table_ld=0) == "AWEQ_ERR_SHAPE"
    assert bad(q=P + 8) == bad(out=P + 8) == bad(ldq=1028) == bad(mask=P + 4) == bad(ws=P + 8) == "AWEQ_ERR_ALIGN"
    need = B.aweq_prefix_attention_ws(6, 8, 2, 128, 3, 4, 100, 128)
    assert need > 0 and bad(ws=None) == bad(ws_bytes=need - 1) == "AWEQ_ERR_WORKSPACE"


def test_kv_keep(B):
    ok = dict(k_cache=P, v_cache=P, k_step=None, v_step=None, cache_dt=B.AWEQ_F16, pages=8, page_size=16, Hk=2, D=64, table=P, table_ld=3, lens=P, q_start=P, B=2, T=9,
              kept=P, kept_ld=4, count=P, change=P, stream=0)
    bad = lambda **k: _refused(B.aweq_kv_keep, ok, **k)
    for name in ("k_cache", "v_cache", "table", "lens", "q_start", "kept", "count", "change"):
        assert bad(**{name: None}) == "AWEQ_ERR_NULL"
    assert bad(cache_dt=B.AWEQ_I8) == bad(cache_dt=B.AWEQ_I8, k_step=P) == "AWEQ_ERR_NULL"
    assert bad(cache_dt=B.AWEQ_F32) == "AWEQ_ERR_DTYPE"
    assert bad(pages=0) == bad(page_size=8) == bad(Hk=0) == bad(Hk=65536) == bad(D=0) == bad(D=264) == bad(D=60) == bad(B=0) == bad(T=0) == bad(table_ld=0) == bad(kept_ld=0) == "AWEQ_ERR_SHAPE"
    assert bad(B=2 ** 20, Hk=64) == "AWEQ_ERR_SHAPE"
    assert bad(k_cache=P + 8) == bad(table=P + 2) == bad(change=P + 1) == bad(cache_dt=B.AWEQ_I8, k_step=P + 4, v_step=P) == "AWEQ_ERR_ALIGN"
    apart = dict(table=P + 0x1000, lens=P + 0x2000, q_start=P + 0x3000, kept=P + 0x4000, count=P + 0x5000)
    for at in apart.values():
        assert bad(**apart, change=at + 4) == "AWEQ_ERR_ALIGN"
