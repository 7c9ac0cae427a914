"""Attention of drafted tokens in the forms that small batches do not take: very many ranges of keys, keys past the caches, more sequences than are ordered by their lengths."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_tree_attention import B, Case  # noqa: E402,F401


def parts(B, c, max_len=None, max_q=None):
    """Ranges of keys that the call joins: what its scratch memory is for."""
    size = B.aweq_prefix_attention_ws(c.T, c.Hq, c.Hk, c.D, len(c.lens), max_q or max(c.new), c.prefix, max_len or max(c.lens))
    return size // (c.T * c.Hq * (c.D * 4 + 8))


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("lens,new,prefix,Hq", [([40000], [2], 0, 2), ([38000], [20], 0, 2), ([40000, 300], [7, 5], 0, 1), ([20000], [3], 20000, 2), ([300, 40000, 7], [40, 3, 7], 0, 1),
                                                ([64], [9], 40000, 4)])
def test_more_than_64_ranges(B, lens, new, prefix, Hq, D, codes):   # noqa: F811
    c = Case("f16" if D != 128 else "bf16", codes, D, Hq, 1, 64, lens, new, prefix, seed=D)
    n = parts(B, c)
    print(f"[tree] {n} parts", flush=True)
    assert n > 64
    c.all(B)
    first, second = c.run(B), c.run(B)
    assert torch.equal(first[0], second[0]) and torch.equal(first[1], second[1])


@pytest.mark.parametrize("kind", ["tree", "any", "none"])
def test_more_than_64_ranges_and_other_masks(B, kind):   # noqa: F811
    for codes in (False, True):
        c = Case("f16", codes, 64, 2, 1, 16, [40000, 40], [6, 30], 0, kind=kind, hide=True)
        assert parts(B, c) > 64
        c.all(B)
        # most of them empty
        c = Case("bf16", codes, 64, 2, 1, 16, [33, 9, 3], [6, 9, 3], 0, kind=kind)
        assert parts(B, c, 60000) > 64
        c.all(B, max_len=60000)


@pytest.mark.parametrize("cache", ["f16", "bf16", "f16_i8"])
@pytest.mark.parametrize("D,Hq,Hk", [(128, 8, 4), (64, 8, 8), (256, 4, 2)])
def test_keys_past_the_caches(B, cache, D, Hq, Hk):   # noqa: F811
    """Few rows for each key head, and more than 192 MB of keys and values that the sequences may have."""
    codes = cache.endswith("i8")
    for lens, new in (([3000, 1, 900, 70], [3, 1, 4, 2]), ([1500, 0, 64], [4, 0, 4])):
        c = Case(cache.split("_")[0], codes, D, Hq, Hk, 32, lens, new, 0, seed=D)
        assert max(new) * Hq // Hk <= 16
        max_len = -(-(201 << 20) // (len(lens) * Hk * 2 * D * (1 if codes else 2)))
        assert max_len < 1 << 29
        c.all(B, max_len=max_len)
    c = Case(cache.split("_")[0], codes, D, Hq, Hk, 16, [700, 90], [4, 3], 0, kind="any", seed=D, hide=True, junk=True)
    c.all(B, max_len=-(-(201 << 20) // (2 * Hk * 2 * D * (1 if codes else 2))))


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("n", [63, 64, 65, 130, 300])
def test_many_sequences(B, n, codes):   # noqa: F811
    """Up to 64 sequences are given out by their lengths, equal ones and empty ones among them."""
    new = [(i * 5) % 4 for i in range(n)]
    lens = [m + ((i * 37) % 11) * 30 for i, m in enumerate(new)]
    for prefix in (0, 300):
        Case("f16", codes, 64, 2, 1, 16, lens, new, prefix, seed=n).all(B)
    new = [9 + i % 20 if i % 7 == 0 else 1 for i in range(n)]           # (as many rows as row tiles hold, for some)
    Case("bf16", codes, 128, 2, 1, 16, [m + (i % 13) * 20 for i, m in enumerate(new)], new, 100, seed=n).all(B)


@pytest.mark.parametrize("lens", [[100] * 64, [0] * 63 + [2], [5, 0, 5, 0], [2 ** 10 - k for k in range(64)], [k for k in range(64)]])
def test_lengths_that_are_equal_or_in_order(B, lens):   # noqa: F811
    for codes in (False, True):
        Case("f16", codes, 64, 2, 2, 16, lens, [min(n, 3) for n in lens], 40, seed=3).all(B, max_len=1100, max_q=3)
