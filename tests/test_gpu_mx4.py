"""Microscaled 4-bit floating point: codes and scales against the definition in 64 bits, the values read back, and the product against a sum in 64 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2311_01305_amd import binding
    binding.load_library()
    return binding


def dt_of(B, name):
    return {"f32": B.AWEQ_F32, "f16": B.AWEQ_F16, "bf16": B.AWEQ_BF16}[name]


def encoded(x):
    """Codes [rows, K] and scales [rows, K / 32] of binary32 values, as the definition says."""
    rows, K = x.shape
    v = x.astype(np.float64).reshape(rows, K // 32, 32)
    finite = np.isfinite(v).all(2)
    most = np.where(finite, np.abs(np.where(np.isfinite(v), v, 0.0)).max(2), 1.0)
    e = np.where(most > 0, np.frexp(most)[1] - 1 - 2, -127)
    e = np.maximum(e, -127)
    y = np.abs(np.where(finite[..., None], v, 0.0)) * np.exp2(-e.astype(np.float64))[..., None]
    # nearest of the eight, a tie to the even code
    d = np.abs(y[..., None] - GRID)
    near = d == d.min(3, keepdims=True)
    odd = np.arange(8) % 2
    code = np.argmin(np.where(near, odd, 9), 3)
    sign = np.signbit(np.where(finite[..., None], v, 0.0))
    code = code + 8 * sign
    code = np.where(finite[..., None], code, 0)
    return code.reshape(rows, K).astype(np.uint8), np.where(finite, e + 127, 255).astype(np.uint8)


def unpacked(codes, scales, rows, K):
    """From the layout that the header defines."""
    panels, groups = -(-K // 128), -(-K // 512)
    c = np.asarray(codes).reshape(panels, rows, 64)
    both = np.stack((c & 15, c >> 4), 3).reshape(panels, rows, 128).transpose(1, 0, 2).reshape(rows, panels * 128)
    assert not both[:, K:].any(), "columns past K are zero"
    s = np.asarray(scales).reshape(groups, rows, 4, 4)          # [group][row][place][panel]
    place = [(b % 2) * 2 + b // 2 for b in range(4)]
    s = s[:, :, place].transpose(1, 0, 3, 2).reshape(rows, groups * 16)
    assert (s[:, K // 32:panels * 4] == 127).all(), "scales past K"
    return both[:, :K], s[:, :K // 32]


def values(codes, scales):
    """What they stand for, in 64 bits."""
    step = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127.0))
    return np.where(codes & 8, -1.0, 1.0) * GRID[codes & 7] * np.repeat(step, 32, 1)


def quantised(B, X, dt, factor=None, ldx=None):
    rows, K = X.shape
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    codes = torch.full((B.aweq_mx4_code_bytes(rows, K),), 0xEE, dtype=torch.uint8, device=DEV)
    scales = torch.full((B.aweq_mx4_scale_bytes(rows, K),), 0xEE, dtype=torch.uint8, device=DEV)
    B.aweq_quant_mx4(X, dt_of(B, dt), rows, K, ldx or X.stride(0), factor, codes, scales, status)
    return codes, scales, int(status.item())


def same_codes(got, want, scales):
    """To the bit, the signs of zeros among them."""
    assert np.array_equal(got, want), np.argwhere(got != want)[:5]


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,K,fold", [(1, 32, False), (3, 96, True), (17, 128, True), (16, 160, False), (5, 544, True), (33, 4096, False), (70, 2080, True)])
def test_codes_and_scales(B, dt, rows, K, fold):
    g = torch.Generator(device=DEV)
    g.manual_seed(rows * K)
    ld = K + (8 if dt != "f32" else 4)
    X = torch.full((rows, ld), float("nan"), device=DEV).to(TYPES[dt])
    X[:, :K] = (torch.randn(rows, K, generator=g, device=DEV) * torch.exp(2 * torch.randn(rows, K, generator=g, device=DEV))).to(TYPES[dt])
    X[0, :32] = 0.0
    factor = torch.exp(torch.randn(K, generator=g, device=DEV)) if fold else None
    codes, scales, status = quantised(B, X[:, :K], dt, factor, ld)
    x = X[:, :K].float().cpu().numpy()
    if fold:
        x = x * factor.cpu().numpy()       # one product in binary32
    c, s = unpacked(codes.cpu().numpy(), scales.cpu().numpy(), rows, K)
    wc, wsc = encoded(x)
    assert status == 0 and np.array_equal(s, wsc)
    same_codes(c, wc, s)
    for out_dt in ("f32", "bf16", "f16"):
        out = torch.full((rows, K + 8), 9.0, dtype=TYPES[out_dt], device=DEV)
        B.aweq_mx4_values(codes, scales, rows, K, out, dt_of(B, out_dt), K + 8)
        assert (out[:, K:] == 9.0).all()
        want = torch.from_numpy(values(wc, wsc)).to(TYPES[out_dt])
        assert torch.equal(out[:, :K].cpu(), want)


def test_every_binary16_value(B):
    """Each finite binary16 value, as the largest of a block and as a value below it, at four places in the range of ties."""
    bits = np.arange(65536, dtype=np.uint16)
    v = bits.view(np.float16)
    v = v[np.isfinite(v)]
    X = np.zeros((len(v), 32), dtype=np.float16)
    X[:, 0] = v
    X[:, 5], X[:, 31] = np.float16(1.0), np.roll(v, 777)
    X[::2, 5] = np.float16(0.0)
    codes, scales, status = quantised(B, torch.from_numpy(X).to(DEV), "f16")
    c, s = unpacked(codes.cpu().numpy(), scales.cpu().numpy(), len(v), 32)
    wc, wsc = encoded(X.astype(np.float32))
    assert status == 0 and np.array_equal(s, wsc)
    same_codes(c, wc, s)


def test_ties_and_neighbours_at_every_exponent(B):
    """All quotients that lie at a tie, a unit in the last place beside it, and beyond 6, for every scale that binary32 has."""
    ties = np.array([0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 7.0], dtype=np.float32)
    around = np.concatenate([np.nextafter(ties, np.float32(-1)), ties, np.nextafter(ties, np.float32(9))])
    rows = []
    for e in range(-151, 126):
        x = np.concatenate([around, -around]).astype(np.float64) * 2.0 ** e
        for lead in (4.0, 7.999):          # the block's largest, which sets its scale
            with np.errstate(under="ignore", over="ignore"):
                block = np.concatenate([[lead * 2.0 ** e], x]).astype(np.float32)
            block = block[np.abs(block) <= np.float32(lead * 2.0 ** e)]
            rows.append(np.resize(block, 128))
    X = np.stack(rows)
    X[:, ::32] = X[:, :1]
    codes, scales, status = quantised(B, torch.from_numpy(X).to(DEV), "f32")
    c, s = unpacked(codes.cpu().numpy(), scales.cpu().numpy(), *X.shape)
    wc, wsc = encoded(X)
    assert status == 0 and np.array_equal(s, wsc)
    same_codes(c, wc, s)
    out = torch.empty(*X.shape, device=DEV)
    B.aweq_mx4_values(codes, scales, *X.shape, out, B.AWEQ_F32, X.shape[1])
    assert np.array_equal(out.cpu().numpy().astype(np.float64), values(wc, wsc))


@pytest.mark.parametrize("bad", [float("nan"), -float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_what_is_not_finite(B, dt, bad):
    X = torch.randn(4, 160, device=DEV).to(TYPES[dt])
    X[2, 70] = bad
    codes, scales, status = quantised(B, X, dt)
    assert status == B.ST_NONFINITE
    c, s = unpacked(codes.cpu().numpy(), scales.cpu().numpy(), 4, 160)
    wc, wsc = encoded(X.float().cpu().numpy())
    assert np.array_equal(s, wsc) and np.array_equal(c, wc) and (s == 255).sum() == 1
    out = torch.empty(4, 160, device=DEV)
    B.aweq_mx4_values(codes, scales, 4, 160, out, B.AWEQ_F32, 160)
    assert torch.isnan(out[2, 64:96]).all() and torch.isfinite(out).sum() == 4 * 160 - 32


# ---- the product
def product(B, T, N, K, dt, fold, bias, out_dt, seed=1, given=False, ld_extra=0, change=None, ldo_extra=8):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    X = torch.randn(T, K + ld_extra, generator=g, device=DEV)
    X[:, torch.randint(0, K, (max(1, K // 500),), generator=g, device=DEV)] *= 40.0
    X = X.to(TYPES[dt])
    if change:
        change(X)
    factor = torch.exp(0.5 * torch.randn(K, generator=g, device=DEV)) if fold else None
    b = torch.randn(N, generator=g, device=DEV) if bias else None
    W = torch.randn(N, K, generator=g, device=DEV)
    wq, w_scale, _ = quantised(B, W, "f32")
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    xq, x_scale, _ = quantised(B, X[:, :K], dt, factor, K + ld_extra)
    if not given:
        first = (xq, x_scale)
        xq, x_scale = torch.full_like(xq, 0xEE), torch.full_like(x_scale, 0xEE)
    ldo = N + ldo_extra
    out = torch.full((T, ldo), 5.0, dtype=TYPES[out_dt], device=DEV)
    B.aweq_mx4_gemm_tokens(None if given else X, dt_of(B, dt), T, K, K + ld_extra, factor, xq, x_scale, wq, w_scale, N, b, out, dt_of(B, out_dt), ldo, status)
    assert (out[:, N:] == 5.0).all()
    cx = unpacked(xq.cpu().numpy(), x_scale.cpu().numpy(), T, K)
    if not given:
        want = unpacked(first[0].cpu().numpy(), first[1].cpu().numpy(), T, K)
        assert np.array_equal(cx[0], want[0]) and np.array_equal(cx[1], want[1])
    x = torch.from_numpy(values(*cx))
    w = torch.from_numpy(values(*unpacked(wq.cpu().numpy(), w_scale.cpu().numpy(), N, K)))
    return out[:, :N].double().cpu(), x, w, None if b is None else b.double().cpu(), int(status.item())


def check(out, x, w, b, out_dt):
    """Products of the codes' values are exact.  Within: K additions in fp32 in any order, each off by 2^-23 at most of what has come together (truncated, at worst), which
    is no more than the sum of the sizes; one more for the bias; the output's rounding, and binary16's subnormal step."""
    K = x.shape[1]
    want, sizes = x @ w.t(), x.abs() @ w.abs().t()
    if b is not None:
        want, sizes = want + b, sizes + b.abs()
    unit = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}[out_dt]
    allowed = (K + 1) * 2.0 ** -23 * sizes + unit * want.abs() + (2.0 ** -25 if out_dt == "f16" else 0.0)
    off = (out - want).abs()
    assert (off <= allowed).all(), (float(off.max()), float((off / allowed).max()))
    # and as far as sums of that many roundings come in earnest: their root
    rms = float(((out - want) ** 2).mean().sqrt() / (want ** 2).mean().sqrt())
    assert rms <= unit + 2.0 ** -23 * K ** 0.5 * 4, rms


SIZES = [(1, 4, 32), (1, 64, 4096), (2, 100, 544), (3, 20, 96), (4, 2052, 1056), (5, 36, 2080), (16, 64, 512), (17, 48, 1024), (31, 132, 640), (33, 260, 1536),
         (64, 128, 4608), (65, 516, 128), (100, 1028, 2016), (129, 260, 384), (200, 300, 5152), (257, 516, 1120), (300, 260, 160), (511, 8196, 256), (700, 2100, 1088),
         (130, 1300, 9056), (260, 512, 4160), (1000, 1036, 1440), (2300, 260, 800), (4200, 4100, 1312), (6000, 2052, 928), (900, 9000, 992),
         (1, 64, 32768), (4, 64, 8192), (2, 36, 33024), (70, 132, 33024), (3, 8, 64),
         (3, 6000, 544), (520, 6004, 544), (777, 4100, 1056), (1500, 2052, 1440), (777, 16388, 544),
         (16, 36, 1024), (13, 132, 544), (2, 68, 8192), (16, 5004, 512), (9, 12000, 288), (3, 8, 1 << 20), (40, 4, 1 << 20)]


@pytest.mark.parametrize("T,N,K", SIZES)
@pytest.mark.parametrize("dt,out_dt", [("f16", "f16"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
def test_product(B, T, N, K, dt, out_dt):
    fold, bias = (T + N) % 2 == 0, T % 3 != 0
    print(f"[product] T={T} N={N} K={K} {dt} {out_dt}", flush=True)
    got = product(B, T, N, K, dt, fold, bias, out_dt, seed=T + K, ld_extra=8 * (T % 2))
    assert got[4] == 0
    check(*got[:4], out_dt)


@pytest.mark.parametrize("T,N,K", [(2, 64, 96), (40, 260, 544), (300, 1024, 640), (1500, 1028, 1312)])
@pytest.mark.parametrize("out_dt", ["f16", "f32"])
def test_rows_of_the_output_that_begin_anywhere(B, T, N, K, out_dt):
    """Pitches that are no multiple of 16 bytes' worth, and none at all."""
    for extra in (0, 4, 12):
        got = product(B, T, N, K, "bf16", False, True, out_dt, ldo_extra=extra)
        assert got[4] == 0
        check(*got[:4], out_dt)


@pytest.mark.parametrize("T,N,K", [(1, 100, 544), (9, 260, 2048), (150, 516, 1056), (600, 2100, 640)])
def test_codes_that_are_given(B, T, N, K):
    got = product(B, T, N, K, "f16", True, True, "f32", given=True)
    assert got[4] == 0
    check(*got[:4], "f32")


@pytest.mark.parametrize("T", [1, 4, 20, 200, 700])
def test_tokens_that_are_not_finite(B, T):
    """Their outputs are NaN, and nobody else's."""
    def change(X):
        X[T // 2, 100] = float("inf")
    out, x, w, b, status = product(B, T, 516, 1120, "f16", False, False, "f32", change=change)
    assert status == B.ST_NONFINITE
    assert torch.isnan(out[T // 2]).all()
    rest = torch.arange(T) != T // 2
    if rest.any():
        check(out[rest], x[rest], w, b, "f32")


@pytest.mark.parametrize("T", [1, 20, 200, 700])
def test_weights_that_are_not_finite(B, T):
    """Their channel's outputs are NaN, and no other's."""
    g = torch.Generator(device=DEV)
    g.manual_seed(T)
    N, K = 516, 1120
    W = torch.randn(N, K, generator=g, device=DEV)
    W[77, 1100], W[300, 3] = float("nan"), -float("inf")
    wq, w_scale, status = quantised(B, W, "f32")
    X = torch.randn(T, K, generator=g, device=DEV)
    xq, x_scale, _ = quantised(B, X, "f32")
    out = torch.empty(T, N, device=DEV)
    B.aweq_mx4_gemm_tokens(None, B.AWEQ_F32, T, K, K, None, xq, x_scale, wq, w_scale, N, None, out, B.AWEQ_F32, N)
    bad = torch.zeros(N, dtype=torch.bool)
    bad[77] = bad[300] = True
    assert status == B.ST_NONFINITE and torch.isnan(out[:, bad.to(DEV)]).all()
    x = torch.from_numpy(values(*unpacked(xq.cpu().numpy(), x_scale.cpu().numpy(), T, K)))
    w = torch.from_numpy(values(*unpacked(wq.cpu().numpy(), w_scale.cpu().numpy(), N, K)))
    check(out.double().cpu()[:, ~bad], x, w[~bad], None, "f32")


def test_large_and_small_scales(B):
    """Products between 2^-130 and 2^120: sums that cancel in no way, scales at the ends of their range."""
    T, N, K = 5, 64, 256
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    X = torch.randn(T, K, generator=g, device=DEV) * torch.tensor([2.0 ** -120, 2.0 ** -60, 1.0, 2.0 ** 60, 2.0 ** 100], device=DEV)[:, None]
    W = torch.randn(N, K, generator=g, device=DEV) * 2.0 ** -3
    wq, w_scale, _ = quantised(B, W, "f32")
    xq, x_scale, _ = quantised(B, X, "f32")
    out = torch.empty(T, N, device=DEV)
    B.aweq_mx4_gemm_tokens(None, B.AWEQ_F32, T, K, K, None, xq, x_scale, wq, w_scale, N, None, out, B.AWEQ_F32, N)
    x = torch.from_numpy(values(*unpacked(xq.cpu().numpy(), x_scale.cpu().numpy(), T, K)))
    w = torch.from_numpy(values(*unpacked(wq.cpu().numpy(), w_scale.cpu().numpy(), N, K)))
    check(out[1:].double().cpu(), x[1:], w, None, "f32")
    off = (out[0].double().cpu() - x[:1] @ w.t()).abs()
    assert (off <= K * 2.0 ** -23 * (x[:1].abs() @ w.abs().t()) + K * 2.0 ** -126).all()   # (a matrix unit may take a subnormal sum for 0)


def test_repeats_are_the_same_to_the_bit_and_streams(B):
    for T, N, K in ((3, 516, 2080), (40, 516, 2080), (300, 1028, 2080), (1500, 1028, 544)):
        a = product(B, T, N, K, "bf16", True, True, "f32")[0]
        b = product(B, T, N, K, "bf16", True, True, "f32")[0]
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            c = product(B, T, N, K, "bf16", True, True, "f32")[0]
        side.synchronize()
        assert torch.equal(a, b) and torch.equal(a, c)
