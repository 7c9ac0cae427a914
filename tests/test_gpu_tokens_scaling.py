"""The scaling of the product with a quantizer a token, where binary32 does not hold it: biases that cancel the product, steps whose product is below binary32's
normal numbers, zero points outside the range that a token's can have.  In every form that the sizes lead to."""
import numpy as np
import pytest

from conftest import to_panels

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # half a unit of the last place, relative
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2311_01305_amd import binding
    binding.load_library()
    return binding


# (T, N, K): few tokens in both tiles, quantised by the product and not; some hundred; tiled with either tile, whole and with edges
SHAPES = [(1, 260, 72), (2, 1024, 520), (4, 64, 4096), (5, 68, 200), (17, 4096, 1024), (64, 6148, 512), (130, 1028, 264), (300, 4100, 328), (1000, 4096, 512),
          (2300, 4092, 136), (4100, 1024, 64)]


class Layer:
    def __init__(self, N, K, seed, small=1.0):
        rng = np.random.default_rng(seed)
        self.N, self.K = N, K
        self.codes = rng.integers(-128, 128, (N, K)).astype(np.int8)
        self.step = ((rng.random(N) + 0.5) * 1e-3 * small).astype(np.float32)
        self.zero = rng.integers(0, 256, N).astype(np.int32)
        up = lambda a: torch.from_numpy(a).to(DEV)
        self.d = (up(to_panels(self.codes)), up(self.step), up(self.zero), up(self.codes.astype(np.int64).sum(1).astype(np.int32)))

    def call(self, B, x, dt, out, bias, codes=None):
        """x: values, or (codes) the quantizer's outputs"""
        T, N, K = x.shape[0], self.N, self.K
        kind = {"f32": B.AWEQ_F32, "f16": B.AWEQ_F16, "bf16": B.AWEQ_BF16}
        if codes is None:
            e = lambda n, t: torch.empty(n, dtype=t, device=DEV)
            codes = [e(B.aweq_panel_bytes(T, K), torch.int8), e(T, torch.float32), e(T, torch.int32), e(T, torch.int32)]
            given, kind_x, ld = x, kind[dt], x.stride(0)
        else:
            given, kind_x, ld = codes[0], B.AWEQ_I8, K
        y = torch.empty(T, N, dtype=TYPES[out], device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        wq, sw, zw, rw = self.d
        B.aweq_w8a8_gemm_tokens(given, kind_x, T, K, ld, None, *codes, wq, N, sw, zw, 0, rw, bias, y, kind[out], N, status)
        return y.double(), codes, int(status.item())

    def scaled(self, B, codes, T):
        """The product in 64 bits from the quantizer's outputs: its integer is exact there."""
        panels = codes[0].view(-(-self.K // 64), T, 64).transpose(0, 1).reshape(T, -1)[:, :self.K]
        left = panels.double() + (128.0 - codes[2].double())[:, None]
        right = torch.from_numpy(self.codes).to(DEV).double() + (128.0 - self.d[2].double())[:, None]
        return (left @ right.t()) * codes[1].double()[:, None] * self.d[1].double()[None, :]


@pytest.mark.parametrize("T,N,K", SHAPES)
@pytest.mark.parametrize("dt,out", [("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32")])
def test_biases_that_cancel_the_product(B, T, N, K, dt, out):
    """One token's product is taken off by the bias up to its rounding to binary32: what is left is of that size, and has the output's digits."""
    print(f"[scaling] cancel T={T} N={N} K={K} {dt} -> {out}", flush=True)
    layer = Layer(N, K, T + N)
    x = torch.randn(T, K, device=DEV).to(TYPES[dt])
    _, codes, _ = layer.call(B, x, dt, out, None)
    scaled = layer.scaled(B, codes, T)
    for t in {0, T // 2, T - 1}:
        bias = (-scaled[t]).float()
        y, _, status = layer.call(B, x, dt, out, bias)
        assert status == 0
        want = scaled + bias.double()
        # rounded in 64 bits, to binary32 and to the output's type
        allowed = (UNIT[out] * 1.001 + 2.0 ** -24) * want.abs() + 2.0 ** -50 * scaled.abs() + TINY[out]
        off = (y - want).abs()
        assert bool((off <= allowed).all()), (t, float((off / allowed).max()))


@pytest.mark.parametrize("T,N,K", SHAPES)
def test_steps_whose_product_is_small(B, T, N, K):
    """bfloat16 holds outputs for which the product of the two steps is no normal number of binary32."""
    print(f"[scaling] small T={T} N={N} K={K}", flush=True)
    layer = Layer(N, K, T + N, small=1e-12)
    x = (torch.randn(T, K, device=DEV) * 1e-24).to(torch.bfloat16)
    for out in ("bf16", "f32"):
        y, codes, status = layer.call(B, x, "bf16", out, None)
        assert status == 0
        want = layer.scaled(B, codes, T)
        assert float((codes[1].double().max() * layer.d[1].double().max())) < 2.0 ** -126 < float(want.abs().max())
        allowed = (UNIT[out] * 1.001 + 2.0 ** -24) * want.abs() + TINY[out] + 2.0 ** -149
        assert bool(((y - want).abs() <= allowed).all()), (out, float(((y - want).abs() / allowed).max()))


@pytest.mark.parametrize("T,N,K", SHAPES)
def test_zero_points_that_no_token_can_have(B, T, N, K):
    """Given codes whose zero point is outside [0, 255] are reported and taken as if it were the nearest inside, whatever form the sizes lead to."""
    layer = Layer(N, K, T + N)
    x = torch.randn(T, K, device=DEV).half()
    _, codes, status = layer.call(B, x, "f16", "f16", None)
    assert status == 0
    for zero in (-1, 256, 300, -20000):
        print(f"[scaling] zero T={T} N={N} K={K} {zero}", flush=True)
        outside, inside = codes[2].clone(), codes[2].clone()
        outside[T // 2], inside[T // 2] = zero, min(max(zero, 0), 255)
        y, _, status = layer.call(B, x, "f16", "f32", None, [codes[0], codes[1], outside, codes[3]])
        want, _, none = layer.call(B, x, "f16", "f32", None, [codes[0], codes[1], inside, codes[3]])
        assert status == B.ST_ZEROPOINT and none == 0
        assert torch.equal(y, want)
