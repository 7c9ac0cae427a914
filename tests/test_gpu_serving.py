"""The served attention block: its calls together against the formulas on its own intermediate values, prompts against the same tokens one by one, and
a decode step as a graph."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HIDDEN, HQ, HK, D, PAGE = 256, 4, 2, 64, 16


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2311_01305_amd import serving
    serving.B.load_library()
    return serving


def ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device=DEV)


def block(S, codes=False, dtype=torch.float16, max_tokens=64, pages=64):
    cache = S.PagedCache(pages, PAGE, HK, D, dtype=dtype, codes=codes, device=DEV)
    for t in (cache.k, cache.v):
        t.fill_(0 if codes else float("nan"))
    w = 1 + 0.1 * torch.arange(D, device=DEV).float() / D
    return S.AttentionBlock(S.calibrated((HQ + 2 * HK) * D, HIDDEN, 1), S.calibrated(HIDDEN, HQ * D, 2), HQ, cache, S.frequencies(32, device=DEV), 32, max_tokens,
                            q_norm=w, k_norm=w, device=DEV)


def turned(x, w, pos):
    """x [T, H, D] normed, its first 32 values rotated (half layout)."""
    x = x / torch.sqrt((x * x).mean(2, keepdim=True) + 1e-6) * w
    f = 10000.0 ** (-2.0 * torch.arange(16, dtype=torch.float64) / 32)
    a = (pos.double()[:, None] * f)[:, None, :]
    u, v = x[..., :16], x[..., 16:32]
    return torch.cat((u * a.cos() - v * a.sin(), v * a.cos() + u * a.sin(), x[..., 32:]), 2)


def rms_off(got, want):
    return float((got - want).norm() / want.norm())


# Relative 2-norms: a value rounded to binary16 / bfloat16 is off by at most 2^-11 / 2^-8; q, k (once more for the rotated ones), the probabilities and the
# output are rounded: scores of size around 3 are off by 3 * 3 of that.  Codes: half of 1 / 127 of the largest of 64 values (about 2.5 rms) for keys and values
BOUNDS = {(torch.float16, False): 16 * 2.0 ** -11, (torch.bfloat16, False): 16 * 2.0 ** -8, (torch.float16, True): 16 * 2.0 ** -11 + 4 * 2.5 * 0.5 / 127}


@pytest.mark.parametrize("dtype,codes", list(BOUNDS))
def test_prompts_behind_a_prefix_and_their_next_tokens(S, dtype, codes):
    torch.manual_seed(3)
    b = block(S, codes, dtype)
    cache = b.cache
    prefix = 37
    pages = cache.take(prefix)
    hidden = {}     # of the tokens of each sequence, by their keys and values as the projection left them

    def attend(x, pos, slot, lens, table, q_start, new, keys, **k):
        y = b(x, pos, slot, lens, table, q_start, int(lens.max()), max(new), **k).clone()
        T = x.shape[0]
        qkv = b.qkv[:T].double().cpu()
        q, kk, v = (qkv[:, i:j].reshape(T, -1, D) for i, j in ((0, HQ * D), (HQ * D, (HQ + HK) * D), ((HQ + HK) * D, (HQ + 2 * HK) * D)))
        w, p = b.q_norm.double().cpu(), pos.cpu()
        q, kk = turned(q, w, p), turned(kk, w, p)
        want, t = torch.zeros(T, HQ, D, dtype=torch.float64), 0
        for s, m in enumerate(new):
            for i in range(m):
                keys[s].append((kk[t], v[t]))
                every = keys["prefix"] + keys[s]
                K, V = (torch.stack([e[n] for e in every], 1) for n in (0, 1))      # [Hk, keys, D]
                sc = torch.softmax((q[t].view(HK, HQ // HK, D) @ K.transpose(1, 2)) / math.sqrt(D), 2)
                want[t] = (sc @ V).reshape(HQ, D)
                t += 1
        assert rms_off(b.attended[:T].double().cpu().view(T, HQ, D), want) <= BOUNDS[(dtype, codes)]
        # the output projection of what the attention left
        a = b.attended[:T].float().cpu().numpy() * b.out_layer.inv_s.cpu().numpy()
        lo, hi = a.min(1).clip(max=0), a.max(1).clip(min=0)
        step = torch.from_numpy((hi - lo) / 255)[:, None]
        codes_ = torch.from_numpy(a).div(step).round() * step
        from paper_2311_01305_amd.layout import from_panels
        wq = torch.from_numpy(from_panels(b.out_layer.codes.cpu().numpy(), HIDDEN, HQ * D)).double()
        wd = (wq + 128 - b.out_layer.zero_w.cpu().double()[:, None]) * b.out_layer.step_w.cpu().double()[:, None]
        assert rms_off(y.double().cpu(), codes_.double() @ wd.t()) <= (2.0 ** -10 if dtype == torch.float16 else 2.0 ** -7)
        return y

    keys = {"prefix": [], 0: [], 1: [], 2: []}
    x0 = torch.randn(prefix, HIDDEN, device=DEV).to(dtype)
    attend(x0, ints(list(range(prefix))), ints(cache.slots(pages, 0, prefix), torch.int64), ints([prefix]), ints([pages]), ints([0, prefix]), [prefix], keys)
    keys["prefix"], keys[0] = keys[0], []
    own = [cache.take(40) for _ in range(3)]
    table, shared = ints(own), ints(pages)
    new, lens = [5, 18, 1], [0, 0, 0]
    for round_ in range(4):
        T = sum(new)
        x = torch.randn(T, HIDDEN, device=DEV).to(dtype)
        pos = [prefix + lens[s] + i for s in range(3) for i in range(new[s])]
        slot = [c for s in range(3) for c in cache.slots(own[s], lens[s], new[s])]
        lens = [n + m for n, m in zip(lens, new)]
        start = None if new == [1, 1, 1] else ints([sum(new[:s]) for s in range(4)])
        attend(x, ints(pos), ints(slot, torch.int64), ints(lens), table, start, new, keys, prefix_table=shared, prefix_len=prefix)
        new = [1, 1, 1]
    assert int(b.status.item()) == 0


def test_a_decode_step_as_a_graph(S):
    torch.manual_seed(5)
    b, e = block(S), block(S)
    batch, steps = 3, 5
    own = [b.cache.take(20) for _ in range(batch)]
    for c in (b.cache, e.cache):
        c.k.zero_(), c.v.zero_()
    table = ints(own)
    x = torch.zeros(batch, HIDDEN, dtype=torch.float16, device=DEV)
    pos, slot, lens = ints([0] * batch), ints([0] * batch, torch.int64), ints([0] * batch)
    b.reserve(batch, batch, 1, 0, 20)
    e.reserve(batch, batch, 1, 0, 20)

    def fill(i):
        x.copy_(torch.randn(batch, HIDDEN, device=DEV))
        pos.fill_(i), lens.fill_(i + 1)
        slot.copy_(ints([b.cache.slots(p, i, 1)[0] for p in own], torch.int64))

    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b(x, pos, slot, lens, table, None, 20, 1)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            y = b(x, pos, slot, lens, table, None, 20, 1)
    torch.cuda.current_stream().wait_stream(side)
    for i in range(steps):
        fill(i)
        graph.replay()
        torch.cuda.synchronize()
        want = e(x, pos, slot, lens, table, None, 20, 1)
        torch.cuda.synchronize()
        assert torch.equal(y, want), i


def test_refusals(S):
    b = block(S)
    with pytest.raises(ValueError):
        b(torch.zeros(65, HIDDEN, dtype=torch.float16, device=DEV), None, None, ints([1]), ints([[0]]), None, 1, 1)
    with pytest.raises(ValueError):
        b(torch.zeros(1, HIDDEN, device=DEV), None, None, ints([1]), ints([[0]]), None, 1, 1)
    with pytest.raises(RuntimeError):
        b.cache.take(64 * PAGE + 1)
    with pytest.raises(ValueError):
        S.AttentionBlock(b.out_layer, b.out_layer, HQ, b.cache, None, 0, 4, device=DEV)
