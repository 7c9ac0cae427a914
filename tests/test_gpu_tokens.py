"""Quantizer with a token as its slice, and the int8 product whose tokens carry scales of their own, against plain numpy: codes, Steps, zero points
and sums to the bit, outputs within the roundings that the header states."""
import numpy as np
import pytest

from conftest import from_panels, to_panels

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


TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # half a unit of the last place, relative
TINY = {"f32": 1e-37, "f16": 2.0 ** -24, "bf16": 1e-37}           # and where the type runs out of exponents


def dt_of(B, name):
    return {"f32": B.AWEQ_F32, "f16": B.AWEQ_F16, "bf16": B.AWEQ_BF16}[name]


def activations(rng, T, K, dt, kind="normal"):
    x = rng.standard_normal((T, K)).astype(np.float32)
    x[:, rng.integers(0, K, max(1, K // 500))] *= 40
    if kind == "one_sided":
        x = np.abs(x)
    if kind == "edge":   # tokens of zeros, of one value, of one non-zero value, below 0, of the smallest numbers
        x[0] = 0
        x[1 % T] = 3.0
        x[2 % T] = 0
        x[2 % T, K - 1] = -2.5
        x[3 % T] = -np.abs(x[3 % T])
        x[4 % T] *= 1e-7
    return torch.from_numpy(x).to(TYPES[dt]).to(DEV)


def reference_codes(x, inv_s):
    """Eq. 1-2 in single IEEE operations."""
    a = x * inv_s if inv_s is not None else x
    lo, hi = np.minimum(a.min(1), np.float32(0)), np.maximum(a.max(1), np.float32(0))
    step = ((hi - lo) / np.float32(255)).astype(np.float32)
    step[~(step > 0)] = 1
    zero = np.clip(-np.rint(lo / step), 0, 255).astype(np.int32)
    u = np.clip(np.rint(a / step[:, None]).astype(np.int64) + zero[:, None], 0, 255)
    return (u - 128).astype(np.int8), step, zero


def quantised(B, X, K, fold, rng, dt):
    T = X.shape[0]
    inv_s = np.exp(rng.standard_normal(K) * 0.5).astype(np.float32) if fold else None
    e = lambda n, t: torch.full((n,), 77, dtype=t, device=DEV)
    o = dict(xq=e(B.aweq_panel_bytes(T, K), torch.int8), step=e(T, torch.float32), zero=e(T, torch.int32), rowsum=e(T, torch.int32),
             status=torch.zeros(1, dtype=torch.int32, device=DEV))
    return inv_s, torch.from_numpy(inv_s).to(DEV) if fold else None, o


QUANT = [(1, 8, 8), (1, 4096, 4096), (3, 64, 64), (5, 72, 80), (7, 520, 528), (2, 4104, 4104), (9, 11008, 11008), (4, 16384, 16392), (3, 32768, 32768),
         (130, 1000, 1000), (257, 2048, 2048)]


@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,K,ldx", QUANT)
def test_codes_are_those_of_the_definition(B, T, K, ldx, dt):
    rng = np.random.default_rng(T * 7919 + K)
    for kind, fold in (("normal", True), ("one_sided", False), ("edge", False), ("normal", False)):
        whole = torch.zeros(T, ldx, dtype=TYPES[dt], device=DEV)
        whole[:, :K] = activations(rng, T, K, dt, kind)
        X = whole[:, :K]
        inv_s, inv_d, o = quantised(B, X, K, fold, rng, dt)
        B.aweq_quant_tokens(X, dt_of(B, dt), T, K, ldx, inv_d, o["xq"], o["step"], o["zero"], o["rowsum"], o["status"])
        codes, step, zero = reference_codes(X.float().cpu().numpy(), inv_s)
        assert np.array_equal(o["step"].cpu().numpy(), step), kind
        assert np.array_equal(o["zero"].cpu().numpy(), zero), kind
        got = from_panels(o["xq"].cpu().numpy(), T, K)
        assert np.array_equal(got, codes), (kind, np.argwhere(got != codes)[:4])
        assert np.array_equal(o["rowsum"].cpu().numpy(), codes.astype(np.int64).sum(1)), kind
        assert int(o["status"].item()) == 0


def test_values_that_are_not_finite_are_reported(B):
    X = torch.ones(3, 64, dtype=torch.float16, device=DEV)
    X[1, 5] = float("inf")
    _, _, o = quantised(B, X, 64, False, np.random.default_rng(0), "f16")
    B.aweq_quant_tokens(X, B.AWEQ_F16, 3, 64, 64, None, o["xq"], o["step"], o["zero"], o["rowsum"], o["status"])
    assert int(o["status"].item()) == B.ST_NONFINITE
    assert float(o["step"][0]) == float(np.float32(1) / np.float32(255))


def test_range_beyond_binary32(B):
    """hi - lo overflows: Step is formed from its two ends."""
    X = torch.zeros(1, 64, device=DEV)
    X[0, 0], X[0, 1] = 3e38, -3e38
    _, _, o = quantised(B, X, 64, False, np.random.default_rng(0), "f32")
    B.aweq_quant_tokens(X, B.AWEQ_F32, 1, 64, 64, None, o["xq"], o["step"], o["zero"], o["rowsum"], o["status"])
    assert abs(float(o["step"][0]) - 6e38 / 255) <= 1e-6 * 6e38 / 255
    c = from_panels(o["xq"].cpu().numpy(), 1, 64)[0]
    assert c[0] == 127 and c[1] == -128 and int(o["zero"][0]) == 128


# (T, N, K): every form of the product: one to four tokens, few, some hundred, tiled with either tile, edges in both directions
SHAPES = [(1, 4, 8), (1, 260, 72), (1, 4096, 4096), (2, 1024, 520), (3, 516, 1032), (4, 64, 16384), (5, 68, 200), (17, 4096, 1024), (33, 12, 4096), (64, 6148, 512),
          (65, 256, 256), (130, 1028, 264), (200, 4096, 640), (300, 4100, 328), (700, 2048, 384), (1000, 4096, 512), (2300, 4092, 136), (3515, 4468, 72),
          (4100, 1024, 64)]


def product(B, T, N, K, dt, out, fold, bias, group, seed, given=False, zeros="inside", pad=0):
    rng = np.random.default_rng(seed)
    X = activations(rng, T, K, dt, "edge" if seed % 3 == 0 else "normal")
    inv_s, inv_d, o = quantised(B, X, K, fold, rng, dt)
    wq = rng.integers(-128, 128, (N, K)).astype(np.int8)
    n = N if group == 0 else 1
    step_w = (rng.random(n) * 0.01 + 1e-4).astype(np.float32)
    zero_w = rng.integers(0, 256, n).astype(np.int32)
    if zeros == "outside":   # channels whose range does not contain 0
        zero_w = rng.integers(-20000, 20000, n).astype(np.int32)
    b = rng.standard_normal(N).astype(np.float32) if bias else None
    up = lambda a: None if a is None else torch.from_numpy(a).to(DEV)
    wp, sw, zw, rw, bd = up(to_panels(wq)), up(step_w), up(zero_w), up(wq.astype(np.int64).sum(1).astype(np.int32)), up(b)
    ld = N + pad
    y = torch.full((T, ld), -7.0, dtype=TYPES[out], device=DEV)
    x = X.float().cpu().numpy()
    codes, step, zero = reference_codes(x, inv_s)
    if given:
        o["xq"][:] = up(to_panels(codes))
        o["step"][:], o["zero"][:], o["rowsum"][:] = up(step), up(zero), up(codes.astype(np.int64).sum(1).astype(np.int32))
        B.aweq_w8a8_gemm_tokens(o["xq"], B.AWEQ_I8, T, K, K, None, None, o["step"], o["zero"], o["rowsum"], wp, N, sw, zw, group, rw, bd, y,
                                dt_of(B, out), ld, o["status"])
    else:
        B.aweq_w8a8_gemm_tokens(X, dt_of(B, dt), T, K, K, inv_d, o["xq"], o["step"], o["zero"], o["rowsum"], wp, N, sw, zw, group, rw, bd, y,
                                dt_of(B, out), ld, o["status"])
        assert np.array_equal(from_panels(o["xq"].cpu().numpy(), T, K), codes)
        assert np.array_equal(o["step"].cpu().numpy(), step) and np.array_equal(o["zero"].cpu().numpy(), zero)
        assert np.array_equal(o["rowsum"].cpu().numpy(), codes.astype(np.int64).sum(1))
    got = y.cpu().double().numpy()
    assert (got[:, N:] == -7.0).all()
    # the integer in 64 bits on the device's float64 product (exact: below 2^53)
    left = up(codes.astype(np.float64) + (128.0 - zero[:, None]))
    right = up(wq.astype(np.float64)) + (128.0 - zw.double()).expand(N)[:, None]
    whole = (left @ right.t()).cpu().numpy()
    scaled = whole * step.astype(np.float64)[:, None] * np.broadcast_to(step_w.astype(np.float64), (N,))[None, :]
    want = scaled + (b if b is not None else 0.0)
    # three fp32 roundings of the scaled integer and the sum at most, then the output's own
    allowed = UNIT[out] * 1.001 * np.abs(want) + 2.0 ** -22 * np.abs(scaled) + 2.0 ** -22 * np.abs(want) * (out != "f32") + TINY[out]
    if out == "f32":
        allowed = 2.0 ** -23 * np.abs(want) + 1e-12 * np.abs(scaled) + TINY[out]
    assert np.abs(whole).max() < 2 ** 31
    off = np.abs(got[:, :N] - want)
    assert (off <= allowed).all(), (off.max(), np.argwhere(off > allowed)[:4])
    return int(o["status"].item())


@pytest.mark.parametrize("T,N,K", SHAPES)
@pytest.mark.parametrize("dt,out", [("f16", "f16"), ("bf16", "bf16"), ("f32", "f32")])
def test_product(B, T, N, K, dt, out):
    print(f"[tokens] product T={T} N={N} K={K} {dt} -> {out}", flush=True)
    assert product(B, T, N, K, dt, out, fold=T % 2 == 0, bias=T % 3 == 0, group=0, seed=T * 31 + N + K, pad=4 * (T % 2)) == 0


@pytest.mark.parametrize("T,N,K", [(1, 256, 512), (6, 256, 512), (260, 512, 256), (1500, 1024, 192)])
def test_product_of_given_codes_and_other_types(B, T, N, K):
    for dt, out, group in (("f16", "f32", 0), ("bf16", "f16", -1), ("f32", "bf16", 0), ("f16", "f16", -1)):
        assert product(B, T, N, K, dt, out, True, True, group, seed=T + group, given=True) == 0
        assert product(B, T, N, K, dt, out, True, True, group, seed=T + group) == 0


@pytest.mark.parametrize("T,N,K", [(2, 256, 512), (40, 256, 512), (260, 512, 256), (2300, 1024, 192)])
def test_weights_whose_range_does_not_contain_zero(B, T, N, K):
    assert product(B, T, N, K, "f16", "f16", False, False, 0, seed=T, zeros="outside") == B.ST_ZEROPOINT


def test_product_on_another_stream_and_in_a_graph(B):
    T, N, K = 37, 512, 256
    rng = np.random.default_rng(5)
    X = activations(rng, T, K, "f16")
    _, _, o = quantised(B, X, K, False, rng, "f16")
    wq = torch.from_numpy(to_panels(rng.integers(-128, 128, (N, K)).astype(np.int8))).to(DEV)
    sw, zw = torch.rand(N, device=DEV), torch.randint(0, 256, (N,), dtype=torch.int32, device=DEV)
    rw = torch.randint(-1000, 1000, (N,), dtype=torch.int32, device=DEV)
    y, z = (torch.zeros(T, N, dtype=torch.float16, device=DEV) for _ in range(2))
    scaled = sw * 1e-3
    call = lambda out: B.aweq_w8a8_gemm_tokens(X, B.AWEQ_F16, T, K, K, None, o["xq"], o["step"], o["zero"], o["rowsum"], wq, N, scaled, zw, 0, rw, None, out,
                                               B.AWEQ_F16, N, o["status"])
    call(y)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call(z)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call(z)
    side.synchronize()
    assert torch.equal(y, z)
    for _ in range(4):
        X.copy_(activations(rng, T, K, "f16"))
        z.zero_()
        graph.replay()
        torch.cuda.synchronize()
        call(y)
        torch.cuda.synchronize()
        assert torch.equal(y, z)
