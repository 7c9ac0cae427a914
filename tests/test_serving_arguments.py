"""What the served block refuses before anything of it is run: tensors of another type, shape or layout than the library reads by their addresses."""
import pytest

torch = pytest.importorskip("torch")
HIDDEN, HQ, HK, D, PAGE, T, BATCH = 256, 4, 2, 64, 16, 5, 2


@pytest.fixture(scope="module")
def S():
    from paper_2311_01305_amd import serving
    return serving


@pytest.fixture
def calls(S, monkeypatch):
    """The library's calls that a step makes, in order, instead of the calls."""
    made = []
    for name in ("aweq_w8a8_gemm_tokens", "aweq_kv_append", "aweq_prefix_attention"):
        monkeypatch.setattr(S.B, name, lambda *a, name=name, **k: made.append((name, a)))
    return made


def block(S, **changed):
    layer = lambda N, K: S.QuantLinear(N, K, *[None] * 4)
    ok = dict(qkv=layer((HQ + 2 * HK) * D, HIDDEN), out=layer(HIDDEN, HQ * D), q_heads=HQ, cache=S.PagedCache(8, PAGE, HK, D, device="cpu"),
              freq=torch.ones(16, dtype=torch.float64), rot=32, max_tokens=8, q_norm=torch.ones(D), k_norm=torch.ones(D), device="cpu")
    return S.AttentionBlock(**{**ok, **changed})


def arguments(**changed):
    ints = lambda *s, dtype=torch.int32: torch.zeros(*s, dtype=dtype)
    ok = dict(x=torch.zeros(T, HIDDEN, dtype=torch.float16), pos=ints(T), slot=ints(T, dtype=torch.int64), lens=ints(BATCH), table=ints(BATCH, 3), q_start=ints(BATCH + 1),
              max_len=40, max_q=3, prefix_table=ints(2), prefix_len=20)
    return {**ok, **changed}


def test_a_step_calls_the_library_four_times(S, calls):
    block(S)(**arguments())
    assert [n for n, _ in calls] == ["aweq_w8a8_gemm_tokens", "aweq_kv_append", "aweq_prefix_attention", "aweq_w8a8_gemm_tokens"]
    block(S, rot=0, freq=None)(**arguments(pos=None, prefix_table=None, prefix_len=0, q_start=None))


ints = lambda *s, dtype=torch.int32: torch.zeros(*s, dtype=dtype)
WRONG = {
    "slot of 32 bits": dict(slot=ints(T)), "fewer slots": dict(slot=ints(T - 1, dtype=torch.int64)), "slots with gaps": dict(slot=ints(2 * T, dtype=torch.int64)[::2]),
    "pos of 64 bits": dict(pos=ints(T, dtype=torch.int64)), "no pos": dict(pos=None), "fewer pos": dict(pos=ints(1)),
    "lens of 64 bits": dict(lens=ints(BATCH, dtype=torch.int64)), "lens with gaps": dict(lens=ints(2 * BATCH)[::2]),
    "fewer starts": dict(q_start=ints(BATCH)), "starts of 64 bits": dict(q_start=ints(BATCH + 1, dtype=torch.int64)),
    "fewer rows of pages": dict(table=ints(BATCH - 1, 3)), "pages of 64 bits": dict(table=ints(BATCH, 3, dtype=torch.int64)), "pages across": dict(table=ints(3, BATCH).t()),
    "a prefix of fewer pages": dict(prefix_table=ints(1)), "no prefix": dict(prefix_table=None), "a prefix of 64 bits": dict(prefix_table=ints(2, dtype=torch.int64)),
    "other columns": dict(x=torch.zeros(T, HIDDEN + 8, dtype=torch.float16)), "columns apart": dict(x=torch.zeros(HIDDEN, T, dtype=torch.float16).t()),
    "no token": dict(x=torch.zeros(0, HIDDEN, dtype=torch.float16), pos=ints(0), slot=ints(0, dtype=torch.int64)),
    "more tokens": dict(x=torch.zeros(9, HIDDEN, dtype=torch.float16), pos=ints(9), slot=ints(9, dtype=torch.int64)), "another type": dict(x=torch.zeros(T, HIDDEN)),
}


@pytest.mark.parametrize("what", list(WRONG))
def test_what_a_step_refuses(S, calls, what):
    with pytest.raises(ValueError):
        block(S)(**arguments(**WRONG[what]))
    assert not calls


def test_what_a_block_refuses(S):
    for wrong in (dict(freq=torch.ones(16)), dict(freq=None), dict(freq=torch.ones(15, dtype=torch.float64)), dict(q_norm=torch.ones(D - 1)), dict(k_norm=torch.ones(D).half())):
        with pytest.raises(ValueError):
            block(S, **wrong)


def test_lengths_are_bounded_by_the_pages_of_the_table(S, calls):
    """A view's pitch says nothing of the pages in its rows."""
    block(S)(**arguments(table=torch.zeros(BATCH, 50, dtype=torch.int32)[:, :2], max_len=700))
    numbers = [v for v in next(a for n, a in calls if n == "aweq_prefix_attention") if isinstance(v, int)]
    assert 2 * PAGE in numbers and 700 not in numbers


@pytest.mark.parametrize("which", ["x", "pos", "slot", "lens", "table", "q_start", "prefix_table"])
def test_tensors_elsewhere_are_refused(S, calls, which):
    """Their addresses mean nothing to the GPU that the cache is on (here: tensors without memory beside those of the CPU)."""
    with pytest.raises(ValueError):
        block(S)(**arguments(**{which: arguments()[which].to("meta")}))
    assert not calls


def test_a_block_refuses_tensors_elsewhere(S):
    for wrong in (dict(freq=torch.ones(16, dtype=torch.float64, device="meta")), dict(q_norm=torch.ones(D, device="meta")), dict(k_norm=torch.ones(D, device="meta"))):
        with pytest.raises(ValueError):
            block(S, **wrong)


@pytest.mark.parametrize("heads,key_heads,size", [(4, 2, 96), (4, 2, 80), (4, 2, 32), (4, 3, 64)])
def test_heads_that_the_attention_does_not_read(S, heads, key_heads, size):
    """Refused when the block is made, not after a step has filled its cache."""
    layer = lambda N, K: S.QuantLinear(N, K, *[None] * 4)
    with pytest.raises(ValueError):
        S.AttentionBlock(layer((heads + 2 * key_heads) * size, HIDDEN), layer(HIDDEN, heads * size), heads, S.PagedCache(8, PAGE, key_heads, size, device="cpu"), None, 0, 8,
                         device="cpu")
