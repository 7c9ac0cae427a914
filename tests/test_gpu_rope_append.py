"""Norm and rotation of queries and keys, and their way into the paged cache, against the formulas in 64 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 1e-37, "f16": 2.0 ** -24, "bf16": 1e-37}
EPS = 1e-6
# before the output's rounding: the norm's sum (up to 20 additions deep) and root, the angle (2^-25 of a turn), sine and cosine, three
# operations: below 4e-6 of |a| + |b|
WITHIN = 4e-6


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2311_01305_amd import binding
    binding.load_library()
    return binding


def dt_of(B, name):
    return {"f32": B.AWEQ_F32, "f16": B.AWEQ_F16, "bf16": B.AWEQ_BF16}[name]


def turned(x, w, pos, freq, rot, interleaved, gain):
    """x [T, H, D] in 64 bits -> (normed and rotated, |a| + |b| of each value's pair)."""
    y = x.astype(np.float64)
    if w is not None:
        y = y / np.sqrt((y * y).mean(2, keepdims=True) + EPS) * w.astype(np.float64)
    out, size = y.copy(), np.abs(y)
    if rot:
        angle = pos.astype(np.float64)[:, None] * freq[None, :]
        c, s = gain * np.cos(angle)[:, None, :], gain * np.sin(angle)[:, None, :]
        first = slice(0, rot, 2) if interleaved else slice(0, rot // 2)
        second = slice(1, rot, 2) if interleaved else slice(rot // 2, rot)
        a, b = y[:, :, first].copy(), y[:, :, second].copy()
        out[:, :, first], out[:, :, second] = a * c - b * s, b * c + a * s
        both = max(gain, 1.0) * (np.abs(a) + np.abs(b))
        size[:, :, first], size[:, :, second] = both, both
    return out, size


def rows(rng, T, H, D, ld, dt):
    whole = torch.full((T, ld), 9.0, dtype=TYPES[dt], device=DEV)
    whole[:, :H * D] = torch.from_numpy(rng.standard_normal((T, H * D)) * 2).to(TYPES[dt]).to(DEV)
    return whole, whole[:, :H * D].float().cpu().numpy().reshape(T, H, D)


def near(got, want, size, dt):
    allowed = UNIT[dt] * 1.01 * np.abs(want) + WITHIN * size + TINY[dt]
    off = np.abs(got.astype(np.float64) - want)
    assert (off <= allowed).all(), (off.max(), np.argwhere(off > allowed)[:4])


def angles(B, rng, T, rot, kind=0):
    pos = rng.integers(0, 131072, T).astype(np.int32)
    if T > 2:
        pos[0], pos[1], pos[2] = 0, -5, 2 ** 31 - 1
    freq = np.zeros(max(1, rot // 2))
    if rot:
        B.aweq_rope_frequencies(rot, 10000.0, freq, kind if rot > 2 else 0, 8.0, 4096.0, 1.0, 4.0)
    return pos, torch.from_numpy(pos).to(DEV), freq[:rot // 2], torch.from_numpy(freq).to(DEV)


# (T, Hq, Hk, D, rot, interleaved)
SHAPES = [(1, 1, 1, 8, 8, 1), (1, 32, 8, 128, 128, 0), (3, 5, 3, 24, 16, 0), (7, 32, 8, 128, 64, 1), (2, 3, 1, 96, 96, 0), (5, 7, 7, 80, 32, 0), (4, 9, 2, 64, 64, 1),
          (6, 33, 5, 256, 256, 0), (6, 12, 4, 256, 64, 1), (11, 40, 40, 128, 0, 0), (300, 3, 2, 40, 40, 1), (515, 64, 8, 128, 128, 0), (9000, 2, 1, 64, 32, 0)]


@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,Hq,Hk,D,rot,interleaved", SHAPES)
def test_norm_and_rotation(B, T, Hq, Hk, D, rot, interleaved, dt):
    print(f"[rope] T={T} Hq={Hq} Hk={Hk} D={D} rot={rot} {interleaved} {dt}", flush=True)
    rng = np.random.default_rng(T + 13 * D)
    pos, pos_d, freq, freq_d = angles(B, rng, T, rot, T % 4)
    for norm in (True, False):
        ldq, ldk, ldqo, ldko = Hq * D + 8, Hk * D + 16, Hq * D + 24, Hk * D
        q, qn = rows(rng, T, Hq, D, ldq, dt)
        k, kn = rows(rng, T, Hk, D, ldk, dt)
        if norm:
            qn[0, 0] = 0
            q[0, :D] = 0      # a head of zeros
        wq, wk = (rng.random(D).astype(np.float32) + 0.5 for _ in range(2)) if norm else (None, None)
        up = lambda a: None if a is None else torch.from_numpy(a).to(DEV)
        wqd, wkd = up(wq), up(wk)
        qo, ko = (torch.full((T, ld), 5.0, dtype=TYPES[dt], device=DEV) for ld in (ldqo, ldko))
        gain = 1.25 if T % 2 else 1.0
        B.aweq_qk_rope(q, k, dt_of(B, dt), T, Hq, Hk, D, ldq, ldk, pos_d, freq_d, rot, interleaved, gain, wqd, wkd, EPS, qo, ldqo, ko, ldko)
        near(qo[:, :Hq * D].float().cpu().numpy().reshape(T, Hq, D), *turned(qn, wq, pos, freq, rot, interleaved, gain), dt)
        near(ko.float().cpu().numpy().reshape(T, Hk, D), *turned(kn, wk, pos, freq, rot, interleaved, gain), dt)
        assert (qo[:, Hq * D:] == 5.0).all() and (q[:, Hq * D:] == 9.0).all()
        # in place, and one of the two alone
        B.aweq_qk_rope(q, None, dt_of(B, dt), T, Hq, 0, D, ldq, 0, pos_d, freq_d, rot, interleaved, gain, wqd, None, EPS, q, ldq, None, 0)
        B.aweq_qk_rope(None, k, dt_of(B, dt), T, 0, Hk, D, 0, ldk, pos_d, freq_d, rot, interleaved, gain, None, wkd, EPS, None, 0, k, ldk)
        assert torch.equal(q[:, :Hq * D], qo[:, :Hq * D]) and torch.equal(k[:, :Hk * D], ko)
        assert (q[:, Hq * D:] == 9.0).all() and (k[:, Hk * D:] == 9.0).all()


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("T,Hq,Hk,D,rot,interleaved", SHAPES)
def test_append(B, T, Hq, Hk, D, rot, interleaved, codes, dt):
    print(f"[append] T={T} Hq={Hq} Hk={Hk} D={D} rot={rot} {interleaved} {dt} codes={codes}", flush=True)
    rng = np.random.default_rng(T + 7 * D + codes)
    page = (16, 32, 64, 128, 256)[T % 5]
    pages = -(-T // page) + 3
    norm = T % 2 == 1
    pos, pos_d, freq, freq_d = angles(B, rng, T, rot, T % 4)
    ld = (Hq + 2 * Hk) * D
    x, xn = rows(rng, T, Hq + 2 * Hk, D, ld, dt)
    q, k, v = x[:, :Hq * D], x[:, Hq * D:(Hq + Hk) * D], x[:, (Hq + Hk) * D:]
    if T > 3:
        x[3, (Hq + Hk) * D:(Hq + Hk + 1) * D] = 0   # a value head of zeros: Step 1
        xn[3, Hq + Hk] = 0
    wq, wk = (rng.random(D).astype(np.float32) + 0.5 for _ in range(2)) if norm else (None, None)
    up = lambda a: None if a is None else torch.from_numpy(a).to(DEV)
    wqd, wkd = up(wq), up(wk)
    slot = rng.permutation(pages * page)[:T].astype(np.int64)
    left_out = T > 4
    if left_out:
        slot[1], slot[4] = -1, pages * page   # a padded token, and one past the last page
    kind = torch.int8 if codes else TYPES[dt]
    kc, vc = (torch.full((pages, Hk, page, D), 3, dtype=kind, device=DEV) for _ in range(2))
    ks, vs = (torch.full((pages, Hk, page), -2.0, device=DEV) for _ in range(2)) if codes else (None, None)
    qo = torch.empty(T, Hq * D, dtype=TYPES[dt], device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    slot_d = torch.from_numpy(slot).to(DEV)
    B.aweq_kv_append(q, k, v, dt_of(B, dt), T, Hq, Hk, D, ld, ld, ld, pos_d, freq_d, rot, interleaved, 1.0, wqd, wkd, EPS, qo, Hq * D, kc, vc, ks, vs,
                     B.AWEQ_I8 if codes else dt_of(B, dt), pages, page, slot_d, status)
    near(qo.float().cpu().numpy().reshape(T, Hq, D), *turned(xn[:, :Hq], wq, pos, freq, rot, interleaved, 1.0), dt)
    assert int(status.item()) == (B.ST_INDEX if left_out else 0)
    put = np.array([0 <= s < pages * page for s in slot])
    at, row = slot[put] // page, slot[put] % page
    untouched = np.ones((pages, page), bool)
    untouched[at, row] = False
    for cache, steps, want, size in ((kc, ks, *turned(xn[:, Hq:Hq + Hk], wk, pos, freq, rot, interleaved, 1.0)),
                                     (vc, vs, xn[:, Hq + Hk:].astype(np.float64), np.zeros_like(xn[:, Hq + Hk:]))):
        got = cache.float().cpu().numpy().transpose(0, 2, 1, 3)    # [page, row, head, D]
        assert (got[untouched] == 3).all()
        if not codes:
            near(got[at, row], want[put], size[put], dt)
            continue
        step = steps.cpu().numpy().transpose(0, 2, 1)
        assert (step[untouched] == -2.0).all()
        step = step[at, row].astype(np.float64)
        largest = np.abs(want[put]).max(2)
        expected = np.where(largest > 0, largest / 127, 1.0)
        assert (np.abs(step - expected) <= 2 * WITHIN * expected).all()
        assert np.abs(got[at, row]).max() <= 127
        # half a step, and what the value was off before
        off = np.abs(got[at, row] * step[..., None] - want[put])
        assert (off <= 0.5 * step[..., None] * (1 + 1e-5) + 2 * WITHIN * size[put] + 1e-6 * np.abs(want[put])).all(), off.max()
    # without queries: the same cache
    k2, v2 = torch.full_like(kc, 3), torch.full_like(vc, 3)
    B.aweq_kv_append(None, k, v, dt_of(B, dt), T, 0, Hk, D, 0, ld, ld, pos_d, freq_d, rot, interleaved, 1.0, None, wkd, EPS, None, 0, k2, v2, ks, vs,
                     B.AWEQ_I8 if codes else dt_of(B, dt), pages, page, slot_d, status)
    assert torch.equal(k2, kc) and torch.equal(v2, vc)


def test_cache_past_32_bits(B):
    """A slot whose byte offset needs more than 32 bits."""
    Hk, D, page = 8, 128, 256
    pages = 9000                                     # 4.7 GB each for keys and values
    kc, vc = (torch.zeros(pages, Hk, page, D, dtype=torch.float16, device=DEV) for _ in range(2))
    x = torch.randn(2, 3 * Hk * D, device=DEV).half()
    k, v = x[:, Hk * D:2 * Hk * D], x[:, 2 * Hk * D:]
    slot = torch.tensor([pages * page - 1, 5], dtype=torch.int64, device=DEV)
    B.aweq_kv_append(None, k, v, B.AWEQ_F16, 2, 0, Hk, D, 0, 3 * Hk * D, 3 * Hk * D, None, None, 0, 0, 1.0, None, None, EPS, None, 0, kc, vc, None, None, B.AWEQ_F16,
                     pages, page, slot)
    for t, (p, r) in enumerate(((pages - 1, page - 1), (0, 5))):
        assert torch.equal(kc[p, :, r].flatten(), k[t]) and torch.equal(vc[p, :, r].flatten(), v[t])
    assert int((kc != 0).sum()) <= 2 * Hk * D
