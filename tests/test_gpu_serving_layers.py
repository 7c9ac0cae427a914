"""Calibrated layers on their way into the served block: their biases against the formula in 64 bits, and those of a group as one layer against each by itself."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2311_01305_amd import serving
    serving.B.load_library()
    return serving


def values(codes, N, K, zero, step):
    """The weight that 8-bit codes in panels of 64 columns stand for: one product in binary32 each, as the stage defines W~."""
    rows = codes.view(-1, N, 64).transpose(0, 1).reshape(N, -1)[:, :K].float()
    return ((rows + (128.0 - zero.float()).expand(N)[:, None]) * step.expand(N)[:, None]).double()


def expected_bias(t, layer, N, K, bias):
    """b - sum_k (W~ - W_hat) E[x_hat]"""
    off = (values(layer["codes"], N, K, layer["zero_w"], layer["step_w"]) - layer["W_hat"].double()) @ t["mu_xhat"].double()
    return (0.0 if bias is None else bias.double()) - off


def near(got, want):
    assert bool(((got.double() - want).abs() <= 2.0 ** -22 * want.abs() + 1e-9).all())


def activations(T, K):
    x = torch.randn(T, K, device=DEV) + 0.5 * torch.randn(K, device=DEV)     # (channels with means of their own)
    x[:, ::37] *= 20
    return x.half()


def product(S, layer, x):
    T, B = x.shape[0], S.B
    e = lambda n, t: torch.empty(n, dtype=t, device=DEV)
    codes = e(B.aweq_panel_bytes(T, layer.K), torch.int8), e(T, torch.float32), e(T, torch.int32), e(T, torch.int32)
    y = torch.empty(T, layer.N, device=DEV)
    B.aweq_w8a8_gemm_tokens(x, B.AWEQ_F16, T, layer.K, x.stride(0), layer.inv_s, *codes, layer.codes, layer.N, layer.step_w, layer.zero_w, layer.w_group, layer.rowsum_w,
                            layer.bias, y, B.AWEQ_F32, layer.N)
    return y


@pytest.mark.parametrize("group", [0, -1])
@pytest.mark.parametrize("with_bias", [False, True])
def test_a_layers_bias(S, with_bias, group):
    from paper_2311_01305_amd import pipeline
    torch.manual_seed(11)
    T, K, N = 300, 520, 132
    x, w = activations(T, K), torch.randn(N, K, device=DEV).half()
    bias = torch.randn(N, device=DEV) if with_bias else None
    buf = pipeline.LayerBuffers(T, K, N, torch.float16, group=group, want_out_i32=False, device=DEV)
    pipeline.calibrate_layer(x, w, bias, buf, forward=False)
    kept = buf.t["bias_out"].clone()
    layer = S.QuantLinear.from_layer(buf, bias=bias)
    near(layer.bias, expected_bias(buf.t, buf.t, N, K, bias))
    assert torch.equal(buf.t["bias_out"], kept)                        # the calibration's own stays as it is
    plain = S.QuantLinear.from_layer(buf, bias=bias, correct=False)
    assert plain.bias is bias
    # and it is added once: the two products differ by the correction
    off = product(S, layer, x) - product(S, plain, x)
    want = expected_bias(buf.t, buf.t, N, K, None)
    assert bool(((off.double() - want[None, :]).abs() <= 2.0 ** -22 * product(S, plain, x).abs().amax()).all())


@pytest.mark.parametrize("which", ["none", "some", "all", "not corrected"])
def test_layers_of_a_group_as_one(S, which):
    from paper_2311_01305_amd import pipeline
    torch.manual_seed(12)
    T, K, Ns, D = 200, 264, (256, 128, 128), 64
    x = activations(T, K)
    ws = [torch.randn(N, K, device=DEV).half() for N in Ns]
    biases = [torch.randn(N, device=DEV) if which in ("all", "not corrected") or (which == "some" and i == 1) else None for i, N in enumerate(Ns)]
    gb = pipeline.GroupBuffers(T, K, Ns, torch.float16, device=DEV)
    pipeline.calibrate_group(x, ws, biases, gb)
    whole = S.QuantLinear.from_group(gb, biases=biases, correct=which != "not corrected")
    parts, first = [], 0
    for p, N, b in zip(gb.per, Ns, biases):
        if which == "not corrected":
            assert torch.equal(whole.bias[first:first + N], b)
        else:
            near(whole.bias[first:first + N], expected_bias(gb.t, p, N, K, b))
        one = S.QuantLinear(N, K, p["codes"], p["step_w"], p["zero_w"], p["rowsum_w"], whole.bias[first:first + N].clone(), gb.t["inv_s"])
        parts.append(product(S, one, x))
        first += N
    assert torch.equal(product(S, whole, x), torch.cat(parts, 1))
    # four query heads and two key heads of 64: what the block wants in one
    cache = S.PagedCache(4, 16, 2, D, device=DEV)
    block = S.AttentionBlock(whole, S.calibrated(K, 4 * D, 2), 4, cache, S.frequencies(D, device=DEV), D, 8, device=DEV)
    ints = lambda v, dtype=torch.int32: torch.tensor(v, dtype=dtype, device=DEV)
    pages = cache.take(3)
    y = block(x[:3], ints([0, 1, 2]), ints(cache.slots(pages, 0, 3), torch.int64), ints([3]), ints([pages]), ints([0, 3]), 3, 3)
    assert y.shape == (3, K) and bool(torch.isfinite(y).all()) and int(block.status.item()) == 0


def test_refusals(S):
    from paper_2311_01305_amd import pipeline
    gb = pipeline.GroupBuffers(8, 64, (64, 64), torch.float16, device=DEV)
    with pytest.raises(ValueError):
        S.QuantLinear.from_group(gb, biases=[None])
    with pytest.raises(ValueError):
        S.QuantLinear.from_layer(pipeline.LayerBuffers(8, 128, 64, torch.float16, bits=4, group=128, w8a8=False, device=DEV))
