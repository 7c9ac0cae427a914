"""The served block's scratch memory, as far as it needs no GPU: what a reservation covers, and that what was handed out stays."""
import gc
import random
import weakref

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def S():
    from paper_2311_01305_amd import serving
    serving.B.load_library()
    return serving


def block(S, Hq, Hk, D, max_tokens=64):
    hidden = 256
    layer = lambda N, K: S.QuantLinear(N, K, *[None] * 4)
    return S.AttentionBlock(layer((Hq + 2 * Hk) * D, hidden), layer(hidden, Hq * D), Hq, S.PagedCache(4, 16, Hk, D, device="cpu"), None, 0, max_tokens, device="cpu")


def test_a_bound_covers_all_smaller_steps(S):
    B = S.B
    # fewer tokens, more ranges; prompts that join nothing, and decode steps that do
    assert B.aweq_prefix_attention_ws(127, 32, 8, 128, 127, 1, 0, 4096) > B.aweq_prefix_attention_ws(128, 32, 8, 128, 128, 1, 0, 4096)
    assert B.aweq_prefix_attention_ws(2048, 32, 32, 128, 4, 512, 2048, 4096) < B.aweq_prefix_attention_ws(64, 32, 32, 128, 64, 1, 2048, 4096)
    rng = random.Random(1)
    size = lambda most: int(round(most ** rng.random()))
    for _ in range(300):
        Hk = rng.choice((1, 2, 8, 32))
        Hq, D = Hk * rng.choice((1, 2, 4, 8, 9)), rng.choice((64, 128, 256))
        batch, max_q, prefix, length = size(256), size(4096), rng.choice((0, size(40000))), rng.choice((0, size(200000)))
        tokens = min(batch * max_q, 8192, ((1 << 24) - 1) // Hq)
        most = B.aweq_prefix_attention_ws_most(tokens, Hq, Hk, D, batch, max_q, prefix, length)
        for _ in range(100):
            b, q, p, n = (rng.choice((x, size(x) if x else 0)) for x in (batch, max_q, prefix, length))
            t = rng.choice((min(b * q, tokens), size(min(b * q, tokens))))
            assert B.aweq_prefix_attention_ws(t, Hq, Hk, D, b, q, p, n) <= most, (t, Hq, Hk, D, b, q, p, n)
        for more in ((tokens + 1, batch + 1, max_q, prefix, length), (tokens, batch, max_q + 5, prefix + 300, length), (tokens, batch, max_q, prefix, length + 500)):
            if more[0] * Hq < 1 << 24:
                assert B.aweq_prefix_attention_ws_most(more[0], Hq, Hk, D, *more[1:]) >= most
    assert B.aweq_prefix_attention_ws_most(0, 8, 2, 128, 3, 4, 100, 128) == 0
    assert B.aweq_prefix_attention_ws_most(8, 8, 2, 128, 8, 1, 0, 128) == 0


def test_a_reservation_covers_smaller_steps(S):
    b = block(S, 32, 8, 128, 128)
    b.reserve(128, 128, 1, 0, 4096)
    for tokens in range(1, 129):
        assert S.B.aweq_prefix_attention_ws(tokens, 32, 8, 128, tokens, 1, 0, 4096) <= b.ws.numel(), tokens


def test_scratch_that_was_handed_out_stays(S):
    b = block(S, 4, 2, 64)
    handed = []
    for length in (1000, 3000, 9000, 40000):
        b.reserve(3, 3, 1, 2000, length)
        handed.append((weakref.ref(b.ws), b.ws.data_ptr()))
    gc.collect()
    assert all(r() is not None and r().data_ptr() == at for r, at in handed)
    assert sum(t.numel() for t in b.kept) <= b.ws.numel()
    b.reserve(1, 1, 1, 0, 10)
    assert b.ws.data_ptr() == handed[-1][1]
