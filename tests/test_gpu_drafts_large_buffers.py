"""4-bit projections and drafted tokens where offsets pass 32 bits: the far end of a buffer gives what the same numbers give in a small one."""
import pytest

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


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.empty_cache()


def ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device=DEV)


def quantised(B, X, dt):
    rows, K = X.shape
    codes, scales = (torch.empty(n(rows, K), dtype=torch.uint8, device=DEV) for n in (B.aweq_mx4_code_bytes, B.aweq_mx4_scale_bytes))
    B.aweq_quant_mx4(X, dt, rows, K, K, None, codes, scales)
    return codes, scales


def weight(B, codes, scales, rows, K):
    out = torch.empty(rows, K, device=DEV)
    B.aweq_mx4_values(codes, scales, rows, K, out, B.AWEQ_F32, K)
    return out


def near(out, x, w):
    """Products are exact, sums of K of them in fp32 in any order."""
    want, sizes = x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t()
    assert ((out.double() - want).abs() <= (x.shape[1] + 1) * 2.0 ** -23 * sizes).all()


def test_weight(B):
    N, K = (1 << 20) + 4, 8320                       # 4.4 GB of codes, 17 GB of values
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    W = torch.empty(N, K, dtype=torch.bfloat16, device=DEV)
    for rows in W.split(1 << 17):
        rows.normal_(generator=g)
    wq, w_scale = quantised(B, W, B.AWEQ_BF16)
    last = W[-300:].clone()
    del W
    small = quantised(B, last, B.AWEQ_BF16)
    panels = wq.view(-1, N, 64)[:, -300:]
    assert torch.equal(panels.reshape(-1), small[0]) and torch.equal(w_scale.view(-1, N, 16)[:, -300:].reshape(-1)[:300 * 16 * 16], small[1][:300 * 16 * 16])
    w = weight(B, *small, 300, K)
    for T in (2, 40, 300):                            # each of the forms
        X = torch.randn(T, K, generator=g, device=DEV)
        xq, x_scale = quantised(B, X, B.AWEQ_F32)
        out = torch.empty(T, N, device=DEV)
        B.aweq_mx4_gemm_tokens(X, B.AWEQ_F32, T, K, K, None, xq, x_scale, wq, w_scale, N, None, out, B.AWEQ_F32, N)
        near(out[:, -300:], weight(B, xq, x_scale, T, K), w)


def test_tokens(B):
    T, N, K = (1 << 20) + 3, 2052, 96                 # 8.6 GB of outputs
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    X, W = torch.randn(T, K, generator=g, device=DEV), torch.randn(N, K, generator=g, device=DEV)
    (xq, x_scale), (wq, w_scale) = quantised(B, X, B.AWEQ_F32), quantised(B, W, B.AWEQ_F32)
    out = torch.empty(T, N, device=DEV)
    B.aweq_mx4_gemm_tokens(None, B.AWEQ_F32, T, K, K, None, xq, x_scale, wq, w_scale, N, None, out, B.AWEQ_F32, N)
    w = weight(B, wq, w_scale, N, K)
    near(out[-500:], weight(B, *quantised(B, X[-500:], B.AWEQ_F32), 500, K), w)
    near(out[:500], weight(B, *quantised(B, X[:500], B.AWEQ_F32), 500, K), w)


def test_plan(B):
    pages, size = 2 ** 31 - 1, 256
    stack = torch.empty(pages, dtype=torch.int32, device=DEV)
    stack[:2] = ints([pages - 2, pages - 1])
    table = ints([[pages - 3, -1, -1], [pages - 4, -1, -1]])
    lens, count, starts, pos, slot = ints([0, 0]), ints([0]), ints([0] * 3), ints([0] * 4), ints([0] * 4, torch.int64)
    status = ints([0])
    B.aweq_step_plan(ints([255, 7]), ints([2, 1]), 2, size, pages, table, 3, 3, stack, ints([2]), 0, 4, lens, count, starts, pos, slot, status)
    assert int(status) == 0 and lens.tolist() == [257, 8] and int(count) == 1 and table.tolist() == [[pages - 3, pages - 1, -1], [pages - 4, -1, -1]]
    assert slot.tolist() == [(pages - 3) * size + 255, (pages - 1) * size, (pages - 4) * size + 7, -1] and pos.tolist() == [255, 256, 7, 0]


@pytest.mark.parametrize("codes", [False, True])
def test_cache(B, codes):
    """An accepted path is moved, and attended to, on pages at the end of caches of 10 GB each."""
    Hq, Hk, D, size, T = 8, 8, 128, 128, 12
    pages = 40000 if not codes else 80000
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    store, kind = (torch.int8, B.AWEQ_I8) if codes else (torch.float16, B.AWEQ_F16)
    normal = lambda *s: torch.randn(s, generator=g, device=DEV)
    fill = (lambda *s: (40 * normal(*s)).clamp(-127, 127).to(store)) if codes else (lambda *s: normal(*s).to(store))
    small = [fill(6, Hk, size, D) for _ in range(2)] + [normal(6, Hk, size).abs() * 0.03 if codes else None for _ in range(2)]
    large = []
    for c in small:
        large.append(None if c is None else torch.empty(pages, *c.shape[1:], dtype=c.dtype, device=DEV))
        if c is not None:
            large[-1][-6:] = c
    near_table = [[3, 1, 5], [0, 4, 2]]
    tables = [ints(near_table), ints([[pages - 6 + p for p in row] for row in near_table])]
    lens, starts = ints([300, 135]), ints([0, 7, 12])
    q, mask = normal(T, Hq * D).half(), ints([1, 3, 5, 9, 21, 33, 99, 1, 3, 7, 11, 21], torch.int64).view(T, 1)
    outs = []
    for caches, n, table in ((small, 6, tables[0]), (large, pages, tables[1])):
        status, change, out = ints([0]), ints([0, 0]), torch.empty(T, Hq * D, dtype=torch.float16, device=DEV)
        ws_bytes = B.aweq_prefix_attention_ws(T, Hq, Hk, D, 2, 7, 0, 300)
        ws = torch.empty(max(16, ws_bytes), dtype=torch.uint8, device=DEV)
        B.aweq_tree_attention(q, B.AWEQ_F16, T, Hq, D, Hq * D, *caches, kind, n, size, Hk, None, 0, table, 3, lens, starts, 2, 300, 7, mask, 1, D ** -0.5,
                              out, Hq * D, None, ws, status, ws_bytes=ws_bytes)
        B.aweq_kv_keep(*caches, kind, n, size, Hk, D, table, 3, lens, starts, 2, T, ints([[0, 2, 4, 6], [1, 3, 4, 0]]), 4, ints([4, 3]), change, status)
        assert int(status) == 0 and change.tolist() == [-3, -2]
        outs.append([out] + [None if c is None else c[-6:].clone() for c in caches])
    for a, b in zip(*outs):
        assert a is None or torch.equal(a, b)
