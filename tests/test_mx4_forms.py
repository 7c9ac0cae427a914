"""The 4-bit product's forms: that the tests' shapes reach each of them, and the tiled one where a workgroup has several tiles, whose loads and waits run from one into the next."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}

# Row tiles of 64, 128, 192 and 256 tokens: more tiles of 256 channels than there are compute units, of which some lie inside the output; panels of 128 values, a last one that is
# whole or is not, and every remainder of the groups of four that the loop takes.  (T, N, K) by row tile
TILED = {
    1: [(64, 66056, 2176), (64, 66056, 2208), (64, 66056, 2400), (60, 65800, 2528)],
    2: [(257, 32776, 2176), (257, 32776, 2208), (257, 32776, 2400), (257, 32776, 2560)],
    3: [(385, 32776, 2176), (385, 32776, 2208), (385, 32776, 2400), (257, 49160, 2560)],
    4: [(2049, 12296, 2176), (1025, 24584, 2208), (1537, 16392, 2400), (2049, 12296, 2560), (6000, 4104, 1152), (8200, 3080, 928), (8200, 3080, 608)],
}
SHAPES = [(mi, *s) for mi, shapes in TILED.items() for s in shapes]


@pytest.fixture(scope="module")
def B():
    from paper_2311_01305_amd import binding
    binding.load_library()
    return binding


@pytest.fixture(scope="module")
def gpu(B):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return B


def form(B, T, N, K):
    fn = B.load_library()._ZN4aweq8mx4_formElll       # (aweq::mx4_form, which is none of the library's entry points)
    fn.argtypes, fn.restype = [ctypes.c_int64] * 3, ctypes.c_int
    v = fn(T, N, K)
    return ("few", v // 10 % 10, v % 10) if v < 100 else ("mid", v // 10 % 10) if v < 200 else ("tiled", v // 10 % 10)


def test_the_shapes_reach_their_forms(B):
    for mi, T, N, K in SHAPES:
        assert form(B, T, N, K) == ("tiled", mi), (T, N, K)
        rows = 64 * mi
        assert -(-T // rows) * -(-N // 256) > 256 and (T >= rows or T == 60) and N % 8 == 0
    assert {-(-K // 128) % 4 for _, _, _, K in SHAPES} == {0, 1, 2, 3}


def test_every_form_is_among_the_shapes_of_the_product_tests(B):
    from test_gpu_mx4 import SIZES
    reached = {form(B, *s) for s in SIZES} | {form(B, *s[1:]) for s in SHAPES}
    assert reached == {("few", 1, 1), ("few", 1, 2), ("few", 2, 1), ("few", 2, 2), ("few", 4, 2), ("few", 4, 4), ("mid", 0), ("mid", 1)} | {("tiled", mi) for mi in TILED}


# ---- the tiled form
def quantised(B, X, dt, factor=None):
    rows, K = X.shape
    codes, scales = (torch.empty(n(rows, K), dtype=torch.uint8, device=DEV) for n in (B.aweq_mx4_code_bytes, B.aweq_mx4_scale_bytes))
    B.aweq_quant_mx4(X, dt, rows, K, K, factor, codes, scales)
    return codes, scales


def values(B, codes, scales, rows, K):
    """What the codes stand for (the reading back has tests of its own)."""
    out = torch.empty(rows, K, device=DEV)
    B.aweq_mx4_values(codes, scales, rows, K, out, B.AWEQ_F32, K)
    return out.double()


class Product:
    def __init__(self, B, T, N, K, seed, change=None):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.B, self.T, self.N, self.K = B, T, N, K
        self.X = torch.randn(T, K, generator=g, device=DEV).half()
        self.factor = torch.exp(0.5 * torch.randn(K, generator=g, device=DEV))
        self.bias = torch.randn(N, generator=g, device=DEV)
        W = torch.randn(N, K, generator=g, device=DEV)
        if change:
            change(self.X, W)
        self.wq = quantised(B, W, B.AWEQ_F32)
        self.xq = quantised(B, self.X, B.AWEQ_F16, self.factor)
        self.x, self.w = values(B, *self.xq, T, K), values(B, *self.wq, N, K)

    def run(self, out_dt, bias=True, extra=8, given=False):
        """The product, in a buffer with a row and columns more than it has; returns it and the status."""
        B, T, N, K = self.B, self.T, self.N, self.K
        out = torch.full((T + 1, N + extra), 5.0, dtype=TYPES[out_dt], device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        xq, scales = self.xq if given else (torch.full_like(t, 0xEE) for t in self.xq)
        B.aweq_mx4_gemm_tokens(None if given else self.X, B.AWEQ_F16, T, K, K, self.factor, xq, scales, *self.wq, N, self.bias if bias else None, out,
                               {"f32": B.AWEQ_F32, "f16": B.AWEQ_F16, "bf16": B.AWEQ_BF16}[out_dt], N + extra, status)
        assert bool((out[T] == 5.0).all()) and bool((out[:, N:] == 5.0).all())
        return out[:T, :N], int(status.item())

    def check(self, out, out_dt, bias=True, rows=None, channels=None):
        """Products of the codes' values are exact.  Within: K additions in binary32 in any order, each off by 2^-23 at most of what has come together, which is no
        more than the sum of the sizes; one more for the bias; the output's rounding, and binary16's subnormal step."""
        x, w, b = self.x, self.w, self.bias.double()
        if rows is not None:
            x, out = x[rows], out[rows]
        if channels is not None:
            w, b, out = w[channels], b[channels], out[:, channels]
        want, sizes = x @ w.t(), x.abs() @ w.abs().t()
        if bias:
            want, sizes = want + b, sizes + b.abs()
        unit = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}[out_dt]
        allowed = sizes.mul_((self.K + 1) * 2.0 ** -23).add_(unit * want.abs()).add_(2.0 ** -25 if out_dt == "f16" else 0.0)
        off = (out.double() - want).abs()
        assert bool((off <= allowed).all()), (float(off.max()), float((off / allowed).max()))
        # and as far as sums of that many roundings come in earnest: their root
        assert float((off ** 2).mean().sqrt() / (want ** 2).mean().sqrt()) <= unit + 2.0 ** -23 * self.K ** 0.5 * 4


@pytest.mark.gpu
@pytest.mark.parametrize("mi,T,N,K", SHAPES)
def test_tiles_one_after_the_other(gpu, mi, T, N, K):
    """Outputs of every type, in rows that allow stores of 16 bytes and in rows that do not; repeats, and codes that are given, the same to the bit."""
    p = Product(gpu, T, N, K, T + N + K)
    for out_dt in ("f16", "bf16", "f32"):
        for extra in (8, 4):
            print(f"[tiled] {mi} T={T} N={N} K={K} {out_dt} {extra}", flush=True)
            out, status = p.run(out_dt, extra=extra)
            assert status == 0
            p.check(out, out_dt)
            assert torch.equal(out, p.run(out_dt, extra=extra, given=True)[0]) and torch.equal(out, p.run(out_dt, extra=12 - extra)[0])
    out, status = p.run("f16", bias=False, extra=0)
    p.check(out, "f16", bias=False)


@pytest.mark.gpu
@pytest.mark.parametrize("mi", list(TILED))
def test_another_stream(gpu, mi):
    p = Product(gpu, *TILED[mi][1], seed=mi)
    first = [p.run(t)[0] for t in TYPES]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        second = [p.run(t)[0] for t in TYPES]
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))


@pytest.mark.gpu
@pytest.mark.parametrize("mi", list(TILED))
def test_what_is_not_finite(gpu, mi):
    """A token's outputs and a channel's are NaN, and nobody else's: in a workgroup's first tile and in one that follows."""
    T, N, K = TILED[mi][2]
    tokens, channels = sorted({3, T // 2, T - 1}), [5, N // 2, N - 1]

    def change(X, W):
        X[tokens, K - 1], X[tokens[0], 0] = float("inf"), float("nan")
        W[channels, K - 7], W[channels[0], 100] = float("nan"), -float("inf")
    p = Product(gpu, T, N, K, mi, change)
    out, status = p.run("f32")
    assert status == gpu.ST_NONFINITE
    rows, cols = torch.ones(T, dtype=torch.bool, device=DEV), torch.ones(N, dtype=torch.bool, device=DEV)
    rows[tokens], cols[channels] = False, False
    assert bool(torch.isnan(out[~rows]).all()) and bool(torch.isnan(out[:, ~cols]).all())
    p.check(out, "f32", rows=rows, channels=cols)
