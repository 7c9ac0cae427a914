"""Heads that hold what is not finite, on their way into the paged cache: 8-bit codes cannot say so, their step and the status do; a cache of the values' type holds
them as they are."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
D, HQ, HK, PAGE, ROT = 64, 3, 2, 16, 32


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2311_01305_amd import binding
    binding.load_library()
    return binding


def append(B, x, dt, codes, norm, slot):
    T, row, pages = x.shape[0], (HQ + 2 * HK) * D, -(-x.shape[0] // PAGE) + 1
    q, k, v = x.split([HQ * D, HK * D, HK * D], 1)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    freq = torch.empty(ROT // 2, dtype=torch.float64)
    B.aweq_rope_frequencies(ROT, 10000.0, freq)
    w = torch.ones(D, device=DEV) if norm else None
    new = lambda *s, dtype: torch.zeros(s, dtype=dtype, device=DEV)
    kc, vc = (new(pages, HK, PAGE, D, dtype=torch.int8 if codes else TYPES[dt]) for _ in range(2))
    ks, vs = (new(pages, HK, PAGE, dtype=torch.float32) for _ in range(2)) if codes else (None, None)
    status = new(1, dtype=torch.int32)
    kind = {"f16": B.AWEQ_F16, "bf16": B.AWEQ_BF16}[dt]
    B.aweq_kv_append(q, k, v, kind, T, HQ, HK, D, row, row, row, pos, freq.to(DEV), ROT, 0, 1.0, w, w, 1e-6, torch.empty_like(q).contiguous(), HQ * D, kc, vc, ks, vs,
                     B.AWEQ_I8 if codes else kind, pages, PAGE, slot, status)
    return kc, vc, ks, vs, int(status.item())


# tokens: heads split over workgroups, a token each, several tokens a workgroup
@pytest.mark.parametrize("T", [5, 1500, 20000])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_codes_of_heads_that_are_not_finite(B, dt, norm, T):
    g = torch.Generator(device=DEV)
    g.manual_seed(T)
    x = torch.randn(T, (HQ + 2 * HK) * D, generator=g, device=DEV).to(TYPES[dt])
    slot = torch.arange(T, device=DEV)
    clean = append(B, x, dt, True, norm, slot)
    assert clean[4] == 0
    heads = x.view(T, HQ + 2 * HK, D)
    for at, what in ((3, "nan"), (ROT // 2 + 1, "inf"), (D - 1, "-inf")):
        print(f"[append] T={T} {dt} norm={norm} {what} at {at}", flush=True)
        planted = heads.clone()
        planted[T // 2, HQ, at] = float(what)          # a key's head
        planted[T - 2, HQ + 2 * HK - 1, at] = float(what)   # a value's
        kc, vc, ks, vs, status = append(B, planted.view(T, -1), dt, True, norm, slot)
        assert status == B.ST_NONFINITE
        for codes, steps, clean_codes, clean_steps, t, h in ((kc, ks, clean[0], clean[2], T // 2, 0), (vc, vs, clean[1], clean[3], T - 2, HK - 1)):
            bad = torch.zeros_like(steps, dtype=torch.bool)
            bad[t // PAGE, h, t % PAGE] = True
            assert torch.equal(torch.isnan(steps), bad)
            assert torch.equal(steps[~bad], clean_steps[~bad]) and torch.equal(codes[~bad], clean_codes[~bad])
        # what is left out of the cache says nothing
        out = slot.clone()
        out[T // 2] = out[T - 2] = -1
        assert append(B, planted.view(T, -1), dt, True, norm, out)[4] == 0
        # queries are not coded
        planted = heads.clone()
        planted[T // 2, 1, at] = float(what)
        assert append(B, planted.view(T, -1), dt, True, norm, slot)[4] == 0


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_a_cache_of_the_type_holds_them(B, dt):
    T = 5
    x = torch.randn(T, (HQ + 2 * HK) * D, device=DEV).to(TYPES[dt])
    x[2, HQ * D + 40], x[3, (HQ + HK) * D + 5] = float("nan"), float("-inf")
    kc, vc, _, _, status = append(B, x, dt, False, False, torch.arange(T, device=DEV))
    assert status == 0
    assert bool(torch.isnan(kc[0, 0, 2, 40])) and int(torch.isnan(kc).sum()) == 1
    assert float(vc[0, 0, 3, 5]) == float("-inf") and int((~torch.isfinite(vc)).sum()) == 1
