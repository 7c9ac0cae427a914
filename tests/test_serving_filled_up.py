"""Steps that are filled up with rows which belong to no sequence: what the attention is asked for, and the scratch memory that was reserved for it."""
import pytest

torch = pytest.importorskip("torch")
HIDDEN, HQ, HK, D, PAGE = 256, 32, 8, 64, 16


@pytest.fixture(scope="module")
def S():
    from paper_2311_01305_amd import serving
    serving.B.load_library()
    return serving


@pytest.fixture
def calls(S, monkeypatch):
    made = {}
    for name in ("aweq_w8a8_gemm_tokens", "aweq_kv_append", "aweq_prefix_attention", "aweq_tree_attention"):
        monkeypatch.setattr(S.B, name, lambda *a, name=name, **k: made.setdefault(name, []).append(a))
    return made


ints = lambda *s, dtype=torch.int32: torch.zeros(*s, dtype=dtype)


def step(S, block, T, batch, max_q, max_len, tree):
    mask = ints(T, 1, dtype=torch.int64) if tree else None
    return block(torch.zeros(T, HIDDEN, dtype=torch.float16), None, ints(T, dtype=torch.int64), ints(batch), ints(batch, -(-max_len // PAGE)), ints(batch + 1), max_len, max_q,
                 mask=mask)


def new_block(S, max_tokens):
    layer = lambda N, K: S.QuantLinear(N, K, *[None] * 4)
    return S.AttentionBlock(layer((HQ + 2 * HK) * D, HIDDEN), layer(HIDDEN, HQ * D), HQ, S.PagedCache(4, PAGE, HK, D, device="cpu"), None, 0, max_tokens, device="cpu")


@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("T,batch,max_q,rows", [(20, 2, 3, 6), (6, 2, 3, 6), (5, 2, 3, 5), (64, 1, 1, 1)])
def test_rows_that_no_sequence_can_have_are_not_attended(S, calls, T, batch, max_q, rows, tree):
    y = step(S, new_block(S, 64), T, batch, max_q, 40, tree)
    (call,) = calls["aweq_tree_attention" if tree else "aweq_prefix_attention"]
    assert call[2] == rows and y.shape == (T, HIDDEN)
    assert [a[2] for a in calls["aweq_w8a8_gemm_tokens"]] == [T, T] and calls["aweq_kv_append"][0][4] == T


@pytest.mark.parametrize("tree", [True, False])
def test_a_reservation_covers_filled_up_steps(S, calls, tree):
    """A few tokens of a few sequences in many rows: their keys are split into more ranges, which would be times all rows."""
    assert S.B.aweq_prefix_attention_ws(284, HQ, HK, D, 2, 2, 0, 3828) > S.B.aweq_prefix_attention_ws_most(488, HQ, HK, D, 32, 24, 0, 5000)
    block = new_block(S, 488)
    block.reserve(488, 32, 24, 0, 5000)
    ws = block.ws
    for T in range(1, 489, 7):
        step(S, block, T, 2, 2, 3828, tree)
        step(S, block, T, 5, 1, 5000, tree)
    assert block.ws is ws and not any(k.numel() > 16 for k in block.kept)
