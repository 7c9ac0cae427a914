"""What 4-bit layers, planned steps and steps with masks refuse before anything of them is run, and which calls they make."""
import pytest

torch = pytest.importorskip("torch")
HIDDEN, HQ, HK, D, PAGE, T, BATCH = 256, 4, 2, 64, 16, 6, 2
NAMES = ("aweq_w8a8_gemm_tokens", "aweq_mx4_gemm_tokens", "aweq_quant_mx4", "aweq_kv_append", "aweq_prefix_attention", "aweq_tree_attention", "aweq_step_plan",
         "aweq_tree_mask", "aweq_kv_keep")


@pytest.fixture(scope="module")
def S():
    from paper_2311_01305_amd import serving
    return serving


@pytest.fixture
def calls(S, monkeypatch):
    made = []
    for name in NAMES:
        monkeypatch.setattr(S.B, name, lambda *a, name=name, **k: made.append((name, a)))
    return made


ints = lambda *s, dtype=torch.int32: torch.zeros(*s, dtype=dtype)


def block(S, mx4=True):
    layer = (lambda N, K: S.Mx4Linear.from_weight(torch.zeros(N, K))) if mx4 else (lambda N, K: S.QuantLinear(N, K, *[None] * 4))
    return S.AttentionBlock(layer((HQ + 2 * HK) * D, HIDDEN), layer(HIDDEN, HQ * D), HQ, S.PagedCache(8, PAGE, HK, D, device="cpu"), torch.ones(16, dtype=torch.float64), 32, 8,
                            device="cpu")


def arguments(**changed):
    ok = dict(x=torch.zeros(T, HIDDEN, dtype=torch.float16), pos=ints(T), slot=ints(T, dtype=torch.int64), lens=ints(BATCH), table=ints(BATCH, 3), q_start=ints(BATCH + 1),
              max_len=40, max_q=3, prefix_table=ints(2), prefix_len=20, mask=ints(T, 1, dtype=torch.int64))
    return {**ok, **changed}


def test_calls_of_a_step_with_masks(S, calls):
    block(S)(**arguments())
    assert [n for n, _ in calls][2:] == ["aweq_mx4_gemm_tokens", "aweq_kv_append", "aweq_tree_attention", "aweq_mx4_gemm_tokens"]
    del calls[:]
    block(S, mx4=False)(**arguments(mask=None))
    assert [n for n, _ in calls] == ["aweq_w8a8_gemm_tokens", "aweq_kv_append", "aweq_prefix_attention", "aweq_w8a8_gemm_tokens"]


@pytest.mark.parametrize("wrong", [dict(mask=ints(T, 1)), dict(mask=ints(T - 1, 1, dtype=torch.int64)), dict(mask=ints(T, dtype=torch.int64)),
                                   dict(mask=ints(2, T, dtype=torch.int64).t()), dict(mask=ints(T, 0, dtype=torch.int64)),
                                   dict(q_start=None), dict(mask=ints(T, 1, dtype=torch.int64).to("meta"))])
def test_masks_that_are_refused(S, calls, wrong):
    b = block(S)
    del calls[:]
    with pytest.raises(ValueError):
        b(**arguments(**wrong))
    assert not calls


def test_layers_that_are_refused(S, calls):
    W = torch.zeros(64, 96)
    for wrong in (dict(W=W.t()), dict(W=W[0]), dict(bias=torch.zeros(63)), dict(bias=torch.zeros(64).half()), dict(factor=torch.zeros(95)),
                  dict(factor=torch.zeros(96, dtype=torch.float64)), dict(factor=torch.zeros(192)[::2])):
        with pytest.raises(ValueError):
            S.Mx4Linear.from_weight(**{"W": W, **wrong})
    assert not calls
    layer = S.Mx4Linear.from_weight(W, torch.zeros(64), torch.zeros(96))
    assert (layer.N, layer.K) == (64, 96) and layer.codes.numel() == 64 * 64 and layer.scales.numel() == 64 * 16


def sequences(S, **more):
    return S.Sequences(S.PagedCache(8, PAGE, HK, D, device="cpu"), BATCH, 40, T, **more)


def test_planned_steps(S, calls):
    s = sequences(S)
    assert s.cache.free == [] and int(s.counts[0]) == 8 and tuple(s.table.shape) == (BATCH, 3)
    before, after = s.lengths
    assert s.lens is before
    s.step(ints(BATCH), T)
    assert s.lens is after
    s.draft(ints(T), 64)
    s.keep(ints(BATCH, 2), ints(BATCH), T)
    s.step(s.change, T)
    assert s.lens is before
    assert [n for n, _ in calls] == ["aweq_step_plan", "aweq_tree_mask", "aweq_kv_keep", "aweq_step_plan"]
    s.give_back()
    assert sorted(s.cache.free) == list(range(8)) and int(s.counts[0]) == 0


def test_planned_steps_that_are_refused(S, calls):
    s = sequences(S)
    wrong = [lambda: s.step(ints(BATCH, dtype=torch.int64), T), lambda: s.step(ints(BATCH + 1), T), lambda: s.step(ints(BATCH), 0), lambda: s.step(ints(BATCH), T + 1),
             lambda: s.step(ints(2 * BATCH)[::2], T), lambda: s.draft(ints(T + 1), 3), lambda: s.draft(ints(0), 3), lambda: s.draft(ints(T), 65), lambda: s.draft(ints(T), 0),
             lambda: s.draft(ints(T, dtype=torch.int64), 3), lambda: s.keep(ints(BATCH), ints(BATCH), T), lambda: s.keep(ints(BATCH, 0), ints(BATCH), T),
             lambda: s.keep(ints(BATCH + 1, 2), ints(BATCH), T), lambda: s.keep(ints(BATCH, 2), ints(BATCH, dtype=torch.int64), T), lambda: s.keep(ints(BATCH, 2), ints(BATCH), 0),
             lambda: s.keep(ints(BATCH, 2), ints(BATCH, ).to("meta"), T)]
    for w in wrong:
        with pytest.raises(ValueError):
            w()
    assert not calls and s.at == 0
