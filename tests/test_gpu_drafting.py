"""Steps whose sequences draft trees and keep a path of them, against the same tokens decoded one by one; 4-bit projections; the whole of it captured."""
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


TREES = [[-1, 0, 0, 1, 1, 2, 5], [-1, 0, 1, 2], [-1, -1, 0, 1, 3, 2], [-1]]
PATHS = [[0, 2, 5], [0, 1, 2, 3], [1, 3, 4], [0]]


class Run:
    def __init__(self, S, mx4, codes, prefix, pages=200, seed=3):
        torch.manual_seed(seed)
        self.S, self.prefix = S, prefix
        layers = S.calibrated((HQ + 2 * HK) * D, HIDDEN, 1, mx4=mx4), S.calibrated(HIDDEN, HQ * D, 2, mx4=mx4)
        self.cache = S.PagedCache(pages, PAGE, HK, D, codes=codes, device=DEV)
        self.block = S.AttentionBlock(*layers, HQ, self.cache, S.frequencies(32, device=DEV), 32, 512, device=DEV)
        self.shared = self.cache.take(prefix)
        self.pages = ints(self.shared) if prefix else None
        if prefix:
            x = torch.randn(prefix, HIDDEN, device=DEV).half()
            self.block(x, torch.arange(prefix, dtype=torch.int32, device=DEV), ints(self.cache.slots(self.shared, 0, prefix), torch.int64), ints([prefix]), ints([self.shared]),
                       ints([0, prefix]), prefix, prefix)


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("prefix", [0, 37])
def test_kept_drafts_are_what_decoding_them_gives(S, mx4, codes, prefix):
    """What the attention gives for the kept tokens of every step: keys and values are the same but for a rounding of the projections' sums (2^-11 each, which the score
    multiplies by the query's and the key's size), the probabilities' and the outputs' 2^-11."""
    a, b = Run(S, mx4, codes, prefix), Run(S, mx4, codes, prefix)
    batch = len(TREES)
    seqs = S.Sequences(a.cache, batch, 200, 64, prefix)
    T = sum(map(len, TREES))
    parent = ints([p for t in TREES for p in t])
    more, count = ints([len(t) for t in TREES]), ints([len(p) for p in PATHS])
    kept = ints([p + [0] * (4 - len(p)) for p in PATHS])
    own = [b.cache.take(100) for _ in range(batch)]
    table = ints(own)
    have = [0] * batch
    start = [sum(map(len, TREES[:k])) for k in range(batch)]
    for step in range(6):
        x = torch.randn(T + 2, HIDDEN, device=DEV).half()        # (two rows more than there are tokens)
        q_start, pos, slot = seqs.step(more, T + 2)
        mask = seqs.draft(torch.cat((parent, ints([-1, -1]))), 7)
        a.block(x, pos, slot, seqs.lens, seqs.table, q_start, 200, 7, a.pages, prefix, mask)
        got = a.block.attended[:T].clone()
        seqs.step(seqs.keep(kept, count, T + 2), T + 2)
        for i in range(4):
            # the i-th kept token of each sequence that has one; the others are left out of the cache
            has = [i < len(p) for p in PATHS]
            rows = [start[k] + (PATHS[k][i] if has[k] else 0) for k in range(batch)]
            at = [have[k] + i for k in range(batch)]
            slots = [b.cache.slots(own[k], at[k], 1)[0] if has[k] else -1 for k in range(batch)]
            b.block(x[rows], ints([prefix + n for n in at]), ints(slots, torch.int64), ints([n + 1 if h else 0 for n, h in zip(at, has)]), table, None, 200, 1, b.pages, prefix)
            want = b.block.attended[:batch]
            for k in range(batch):
                if has[k]:
                    w, g = want[k].float(), got[rows[k]].float()
                    assert (g - w).abs().max() <= 2.0 ** -7 * max(1.0, float(w.abs().max())), (step, i, k, float((g - w).abs().max()), float(w.abs().max()))
        have = [n + len(p) for n, p in zip(have, PATHS)]
        assert seqs.lens.tolist() == have
    assert int(seqs.status.item()) == 0 and int(a.block.status.item()) == 0
    # what is not in use is on the stack
    used = sum(-(-n // PAGE) for n in have)
    seqs.give_back()
    held = [p for k in range(batch) for p in seqs.table[k, :-(-have[k] // PAGE)].tolist()]
    assert len(held) == used and sorted(held + a.cache.free + a.shared) == list(range(200))


@pytest.mark.parametrize("codes", [False, True])
def test_captured_steps(S, codes):
    """A step with its drafts, the block, the move of the path and the drop, in one graph: replayed with new inputs between eager work, against eager steps."""
    prefix, batch, m = 300, 3, 9
    runs = [Run(S, True, codes, prefix) for _ in range(2)]
    seqs = [S.Sequences(r.cache, batch, 300, batch * m, prefix) for r in runs]
    x, parent = torch.zeros(batch * m, HIDDEN, dtype=torch.float16, device=DEV), ints([-1] * (batch * m))
    kept, count, more = ints([[0] * 4] * batch), ints([0] * batch), ints([m] * batch)
    for r in runs:
        r.block.reserve(batch * m, batch, m, prefix, 300)

    def step(r, s):
        q_start, pos, slot = s.step(more, batch * m)
        mask = s.draft(parent, m)
        y = r.block(x, pos, slot, s.lens, s.table, q_start, 300, m, r.pages, prefix, mask)
        s.step(s.keep(kept, count, batch * m), batch * m)
        return y

    def fill(i):
        g = torch.Generator()
        g.manual_seed(i)
        x.copy_(torch.randn(batch * m, HIDDEN, generator=g))
        parent.copy_(torch.tensor([-1 if k == 0 else int(torch.randint(-1, k, (1,), generator=g)) for _ in range(batch) for k in range(m)]))
        kept.copy_(torch.stack([torch.randperm(m, generator=g)[:4].sort().values for _ in range(batch)]))
        count.copy_(torch.randint(0, 5, (batch,), generator=g))

    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(runs[0], seqs[0])                      # (eager, once)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            y = step(runs[0], seqs[0])
    torch.cuda.current_stream().wait_stream(side)
    step(runs[1], seqs[1])
    for i in range(1, 9):
        fill(i)
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        want = step(runs[1], seqs[1])
        torch.cuda.synchronize()
        assert torch.equal(got, want), i
        assert torch.equal(seqs[0].lens, seqs[1].lens) and torch.equal(seqs[0].counts[0], seqs[1].counts[0]) and torch.equal(seqs[0].table, seqs[1].table)
        torch.randn(500, 500, device=DEV).sum().item()          # (eager work of the program's own)
    assert all(int(s.status.item()) == 0 for s in seqs) and all(int(r.block.status.item()) == 0 for r in runs)


def test_steps_without_room_change_nothing(S):
    r = Run(S, True, False, 0, pages=6)
    s = S.Sequences(r.cache, 2, 100, 80)
    s.step(ints([40, 30]), 70)
    assert s.lens.tolist() == [40, 30] and int(s.counts[s.at]) == 1
    s.step(ints([20, 20]), 70)
    assert int(s.status.item()) == S.B.ST_PAGES and s.lens.tolist() == [40, 30] and int(s.counts[s.at]) == 1 and s.q_start.tolist() == [0, 0, 0]
    s.step(ints([-40, 20]), 70)
    assert s.lens.tolist() == [0, 50] and int(s.counts[s.at]) == 2


@pytest.mark.parametrize("more", [["--mx4"], ["--draft", "5"], ["--draft", "70", "--mx4", "--codes"]])
@pytest.mark.parametrize("prefix", [0, 70])
def test_command(S, capsys, prefix, more):
    S.main(["--hidden", "256", "--heads", "2", "--key-heads", "1", "--prefix", str(prefix), "--batch", "3", "--steps", "4"] + more)
    out = capsys.readouterr().out
    assert f"behind {prefix} shared tokens" in out and "status 0" in out


@pytest.mark.parametrize("which", ["none", "some", "all"])
def test_layers_of_a_group_as_one(S, which):
    """Each layer's weight as by itself, its bias or zeros, and the whole in a block."""
    from paper_2311_01305_amd import pipeline
    B = S.B
    torch.manual_seed(12)
    T, K, Ns = 200, 288, (256, 128, 128)
    x = torch.randn(T, K, device=DEV).half()
    ws = [torch.randn(N, K, device=DEV).half() for N in Ns]
    biases = [torch.randn(N, device=DEV) if which == "all" or (which == "some" and i == 1) else None for i, N in enumerate(Ns)]
    gb = pipeline.GroupBuffers(T, K, Ns, torch.float16, device=DEV)
    pipeline.calibrate_group(x, ws, biases, gb)
    whole = S.Mx4Linear.from_group(gb, biases=biases)

    def weight(layer):
        out = torch.empty(layer.N, K, device=DEV)
        B.aweq_mx4_values(layer.codes, layer.scales, layer.N, K, out, B.AWEQ_F32, K)
        return out
    assert torch.equal(weight(whole), torch.cat([weight(S.Mx4Linear.from_weight(p["W_hat"])) for p in gb.per]))
    assert whole.factor is gb.t["inv_s"] and (whole.N, whole.K) == (512, K)
    if which == "none":
        assert whole.bias is None
    else:
        assert torch.equal(whole.bias, torch.cat([torch.zeros(N, device=DEV) if b is None else b for N, b in zip(Ns, biases)]))
    with pytest.raises(ValueError):
        S.Mx4Linear.from_group(gb, biases=biases[:2])
    cache = S.PagedCache(4, 16, HK, D, device=DEV)
    block = S.AttentionBlock(whole, S.calibrated(K, HQ * D, 2, mx4=True), HQ, cache, S.frequencies(D, device=DEV), D, 8, device=DEV)
    pages = cache.take(3)
    y = block(x[:3], ints([0, 1, 2]), ints(cache.slots(pages, 0, 3), torch.int64), ints([3]), ints([pages]), ints([0, 3]), 3, 3)
    assert y.shape == (3, K) and bool(torch.isfinite(y).all()) and int(block.status.item()) == 0
