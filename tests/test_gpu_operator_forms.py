"""The forms that the operators take by size where the other tests' sizes do not reach them: many tokens to a workgroup and data past the caches in the
rotation, many parts and data past the caches in the attention, steps next to the smallest numbers."""
import numpy as np
import pytest

from test_gpu_attention import Case
from test_gpu_rope_append import EPS, TINY, UNIT, WITHIN

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2311_01305_amd import binding
    binding.load_library()
    return binding


@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,Hq,Hk,norm,interleaved", [(16400, 3, 1, True, False), (20001, 20, 5, True, False), (33000, 13, 5, False, True), (70001, 2, 1, False, False)])
def test_rotation_of_many_tokens(B, T, Hq, Hk, norm, interleaved, dt):
    """Two to eight tokens a workgroup, the last one with fewer; 150 MB and more (16-bit types) go past the caches."""
    print(f"[forms] rotation T={T} Hq={Hq} Hk={Hk} {dt}", flush=True)
    D, rot, page = 64, 32, 16
    kind = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dt]
    code = {"f32": B.AWEQ_F32, "f16": B.AWEQ_F16, "bf16": B.AWEQ_BF16}[dt]
    g = torch.Generator(device=DEV)
    g.manual_seed(T)
    row = (Hq + 2 * Hk) * D
    x = torch.randn(T, row, generator=g, device=DEV).to(kind)
    q, k, v = x.split([Hq * D, Hk * D, Hk * D], 1)
    pos = torch.randint(0, 100000, (T,), generator=g, device=DEV).to(torch.int32)
    freq = torch.empty(rot // 2, dtype=torch.float64)
    B.aweq_rope_frequencies(rot, 10000.0, freq)
    w = 1 + 0.2 * torch.randn(D, generator=g, device=DEV) if norm else None
    freq = freq.to(DEV)

    def near(got, heads, weight):
        y = heads.unflatten(1, (-1, D)).double()
        if weight is not None:
            y = y / torch.sqrt((y * y).mean(2, keepdim=True) + EPS) * weight.double()
        angle = (pos.double()[:, None] * freq)[:, None, :]
        a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if interleaved else (y[..., :rot // 2], y[..., rot // 2:rot])
        p, s = a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()
        both = a.abs() + b.abs()
        if interleaved:
            want, size = torch.stack((p, s), 3).flatten(2), torch.stack((both, both), 3).flatten(2)
        else:
            want, size = torch.cat((p, s), 2), torch.cat((both, both), 2)
        want, size = torch.cat((want, y[..., rot:]), 2), torch.cat((size, y[..., rot:].abs()), 2)
        off = (got.unflatten(1, (-1, D)).double() - want).abs()
        assert bool((off <= UNIT[dt] * 1.01 * want.abs() + WITHIN * size + TINY[dt]).all()), float(off.max())

    qo, ko = torch.empty(T, Hq * D, dtype=kind, device=DEV), torch.empty(T, Hk * D, dtype=kind, device=DEV)
    B.aweq_qk_rope(q, k, code, T, Hq, Hk, D, row, row, pos, freq, rot, interleaved, 1.0, w, w, EPS, qo, Hq * D, ko, Hk * D)
    near(qo, q, w)
    near(ko, k, w)
    if dt == "f32":
        return
    pages = -(-T // page) + 1
    slot = torch.randperm(pages * page, generator=g, device=DEV)[:T].contiguous()
    kc, vc = (torch.zeros(pages, Hk, page, D, dtype=kind, device=DEV) for _ in range(2))
    q2 = torch.empty_like(qo)
    B.aweq_kv_append(q, k, v, code, T, Hq, Hk, D, row, row, row, pos, freq, rot, interleaved, 1.0, w, w, EPS, q2, Hq * D, kc, vc, None, None, code, pages, page, slot)
    at, r = slot // page, slot % page
    assert torch.equal(q2, qo) and torch.equal(kc[at, :, r].flatten(1), ko) and torch.equal(vc[at, :, r].flatten(1), v)


@pytest.mark.parametrize("cache", ["same", "i8"])
def test_many_parts(B, cache):
    """One sequence with one key head: 71 and 128 ranges, which four wavefronts a row join."""
    for n in (9000, 40001):
        print(f"[forms] one sequence of {n} {cache}", flush=True)
        c = Case("f16", cache, 128, 4, 1, 64, [n], [1], 0, seed=n)
        assert B.aweq_prefix_attention_ws(1, 4, 1, 128, 1, 1, 0, n) > 64 * 4 * 128 * 4
        c.all(B)
    Case("bf16", cache, 64, 2, 1, 16, [9000], [1], 9100, seed=4).all(B)


@pytest.mark.parametrize("cache", ["same", "i8"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_keys_past_the_caches(B, cache, D):
    """A bound of the lengths at which the keys may not fit the caches; and repeats are the same to the bit there."""
    for dt in ("f16", "bf16"):
        c = Case(dt, cache, D, 8, 2, 16, [700, 0, 33, 1500], [1, 1, 1, 1], 0, seed=D)
        c.all(B, max_len=400_000)
        a, b = c.run(B, max_len=400_000), c.run(B, max_len=400_000)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("G", [1, 4, 8])
def test_some_new_tokens_of_each_sequence(B, G):
    """Speculated tokens and chunks of prompts, with and without a prefix: rows of one sequence in tiles of 16, 64 and 128."""
    for m in (2, 3, 16, 17, 40):
        lens, new = [m + 5 * i for i in range(5)], [m - (i % 2) for i in range(5)]
        for prefix in (0, 130):
            print(f"[forms] {m} new tokens x {G}, prefix {prefix}", flush=True)
            Case("f16", "same", 128, 2 * G, 2, 32, lens, new, prefix, seed=m).all(B)
            Case("bf16", "i8", 64, 2 * G, 2, 16, lens, new, prefix, seed=m).all(B)


@pytest.mark.parametrize("dt,cache", [("f16", "same"), ("bf16", "same"), ("f16", "i8")])
@pytest.mark.parametrize("G", [1, 4, 9])
def test_heads_of_256_values(B, G, dt, cache):
    """Their tiles of keys are shorter, and their row tiles another number where single tokens are behind a prefix: ranges that end in each part of a tile."""
    for new in ([1, 1, 1, 1, 1], [1, 0, 20, 3, 1], [40, 33, 0, 64, 1]):
        for prefix in (0, 17, 48, 97, 1100):
            print(f"[forms] heads of 256, x {G}, new {new}, prefix {prefix}", flush=True)
            Case(dt, cache, 256, 2 * G, 2, 16 if prefix % 2 else 128, [n + x for n, x in zip(new, (0, 31, 32, 33, 700))], new, prefix, seed=prefix).all(B)
    Case(dt, cache, 256, 2 * G, 2, 64, [0, 0, 0], [7, 1, 9], 900, seed=G).all(B, max_len=0)


@pytest.mark.parametrize("cache", ["same", "i8"])
@pytest.mark.parametrize("D", [64, 128])
def test_row_tiles_by_the_workgroups_they_leave(B, D, cache):
    """Prompts in tiles of 64 rows (few heads) and of 128 (many), that end in each part of one, and rows of tiles that see different keys."""
    for Hq, Hk, new, before, prefix in ((2, 2, [200, 1, 130], 0, 0), (2, 1, [65, 97], 33, 70), (64, 32, [200, 1, 130], 0, 0), (96, 48, [129, 97, 64], 33, 70)):
        print(f"[forms] row tiles, {Hq}/{Hk} heads of {D} {cache}", flush=True)
        Case("bf16", cache, D, Hq, Hk, 16, [n + before for n in new], new, prefix, seed=Hq).all(B)


def test_steps_next_to_the_smallest_numbers(B):
    """bfloat16 values so small that max / 127 is subnormal: the step stays normal, codes and attention finite."""
    D, page = 64, 16
    x = torch.full((1, 3 * D), 1.5e-38, dtype=torch.bfloat16, device=DEV)
    x[0, 2 * D + 3] = -1.5e-38
    kc, vc = (torch.zeros(1, 1, page, D, dtype=torch.int8, device=DEV) for _ in range(2))
    ks, vs = (torch.zeros(1, 1, page, device=DEV) for _ in range(2))
    slot = torch.zeros(1, dtype=torch.int64, device=DEV)
    B.aweq_kv_append(None, x[:, D:2 * D], x[:, 2 * D:], B.AWEQ_BF16, 1, 0, 1, D, 0, 3 * D, 3 * D, None, None, 0, 0, 1.0, None, None, EPS, None, 0, kc, vc, ks, vs, B.AWEQ_I8, 1,
                     page, slot)
    tiny = np.float32(1.17549435e-38)
    assert float(ks[0, 0, 0]) == tiny and float(vs[0, 0, 0]) == tiny
    assert vc[0, 0, 0].tolist() == [-1 if i == 3 else 1 for i in range(D)]
    out, lse = torch.empty(1, D, dtype=torch.bfloat16, device=DEV), torch.empty(1, 1, device=DEV)
    one = torch.ones(1, dtype=torch.int32, device=DEV)
    B.aweq_prefix_attention(x[:, :D], B.AWEQ_BF16, 1, 1, D, 3 * D, kc, vc, ks, vs, B.AWEQ_I8, 1, page, 1, None, 0, slot.to(torch.int32), 1, one, None, 1, 1, 1, 1.0, out, D, lse, None)
    assert abs(float(lse[0, 0])) <= 1e-5 and bool(torch.isfinite(out).all())
    assert float(out[0, 3]) <= 0 and float(out[0, 0]) >= 0
