"""4-bit quantizer and values of matrices that the caches do not hold, whose forms go past them: to the bit what the same rows give a part at a time."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROWS, K = 12500, 8224          # 206 MB of 16 bits: more than 192, from which the quantizer, and 128, from which the values go past the caches
PARTS = (0, 5000, 9001, ROWS)  # (each less than both)
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2311_01305_amd import binding
    binding.load_library()
    return binding


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.empty_cache()


def kind(B, dt):
    return {"f32": B.AWEQ_F32, "f16": B.AWEQ_F16, "bf16": B.AWEQ_BF16}[dt]


def quantised(B, X, dt, factor):
    rows = X.shape[0]
    codes, scales = (torch.full((n(rows, K),), 0xEE, dtype=torch.uint8, device=DEV) for n in (B.aweq_mx4_code_bytes, B.aweq_mx4_scale_bytes))
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.aweq_quant_mx4(X, kind(B, dt), rows, K, X.stride(0), factor, codes, scales, status)
    return codes.view(-1, rows, 64), scales.view(-1, rows, 16), int(status.item())


@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("fold", [False, True])
def test_quantizer(B, dt, fold):
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    X = torch.randn(ROWS, K + 8, generator=g, device=DEV).to(TYPES[dt])[:, :K]
    X[:, ::97] *= 30.0
    factor = torch.exp(torch.randn(K, generator=g, device=DEV)) if fold else None
    codes, scales, status = quantised(B, X, dt, factor)
    assert status == 0
    used = torch.ones(16, dtype=torch.bool, device=DEV)
    used[3::4] = used[2::4] = used[1::4] = False        # of the last group the first panel's scales (K is 16 groups of 512 and a block)
    for a, b in zip(PARTS, PARTS[1:]):
        c, s, _ = quantised(B, X[a:b], dt, factor)
        assert torch.equal(codes[:, a:b], c) and torch.equal(scales[:-1, a:b], s[:-1]) and torch.equal(scales[-1, a:b][:, used], s[-1][:, used])
    X[ROWS - 1, K - 1] = float("inf")
    codes, scales, status = quantised(B, X, dt, factor)
    assert status == B.ST_NONFINITE and int((scales[:-1] == 255).sum()) == 0 and int((scales[-1][:, used] == 255).sum()) == 1 and int(scales[-1, ROWS - 1, 0]) == 255


@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
def test_values(B, dt):
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    X = torch.randn(ROWS, K, generator=g, device=DEV)
    X[5, 64], X[ROWS - 2, K - 1] = float("nan"), float("inf")
    codes, scales, _ = quantised(B, X, "f32", None)
    del X
    out = torch.full((ROWS, K + 8), 3.0, dtype=TYPES[dt], device=DEV)
    B.aweq_mx4_values(codes, scales, ROWS, K, out, kind(B, dt), K + 8)
    assert bool((out[:, K:] == 3.0).all())
    for a, b in zip(PARTS, PARTS[1:]):
        want = torch.empty(b - a, K, device=DEV)
        B.aweq_mx4_values(codes[:, a:b].contiguous(), scales[:, a:b].contiguous(), b - a, K, want, B.AWEQ_F32, K)
        got, want = out[a:b, :K], want.to(TYPES[dt])
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(nan=7.0), want.nan_to_num(nan=7.0))
    assert int(torch.isnan(out).sum()) == 64
