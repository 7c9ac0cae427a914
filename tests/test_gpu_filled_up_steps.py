"""Steps that are filled up with rows which belong to no sequence: what an earlier, larger step left in the block's buffers has no part in them."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HIDDEN, HQ, HK, D, PAGE, ROWS = 256, 4, 2, 64, 16, 48


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2311_01305_amd import serving
    serving.B.load_library()
    return serving


def ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device=DEV)


class Served:
    """A block with its cache, a prefix in it, and two sequences."""

    def __init__(self, S, mx4, codes, prefix):
        layers = S.calibrated((HQ + 2 * HK) * D, HIDDEN, 1, mx4=mx4), S.calibrated(HIDDEN, HQ * D, 2, mx4=mx4)
        self.cache = S.PagedCache(80, PAGE, HK, D, codes=codes, device=DEV)
        self.block = S.AttentionBlock(*layers, HQ, self.cache, S.frequencies(32, device=DEV), 32, max(ROWS, prefix), device=DEV)
        shared, self.prefix = self.cache.take(prefix), prefix
        self.pages = ints(shared) if prefix else None
        if prefix:
            g = torch.Generator()
            g.manual_seed(9)
            self.block(torch.randn(prefix, HIDDEN, generator=g).half().to(DEV), torch.arange(prefix, dtype=torch.int32, device=DEV),
                       ints(self.cache.slots(shared, 0, prefix), torch.int64), ints([prefix]), ints([shared]), ints([0, prefix]), prefix, prefix)
        self.seqs = S.Sequences(self.cache, 2, 200, ROWS, prefix)
        assert int(self.block.status.item()) == 0

    def step(self, x, more, tree):
        """more: new tokens of each sequence; the rows behind them are nobody's."""
        T = x.shape[0]
        q_start, pos, slot = self.seqs.step(ints(more), T)
        mask = self.seqs.draft(ints([i - 1 for m in more for i in range(m)] + [-1] * (T - sum(more))), max(more)) if tree else None
        return self.block(x, pos, slot, self.seqs.lens, self.seqs.table, q_start, 200, max(more), self.pages, self.prefix, mask)


@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("mx4", [True, False])
@pytest.mark.parametrize("prefix,codes", [(0, False), (300, False), (300, True)])
def test_an_earlier_step_has_no_part_in_the_rows_behind_the_tokens(S, prefix, codes, mx4, tree):
    g = torch.Generator()
    g.manual_seed(prefix)
    x, large = (torch.randn(n, HIDDEN, generator=g).half().to(DEV) for n in (20, ROWS))
    fresh, used = Served(S, mx4, codes, prefix), Served(S, mx4, codes, prefix)
    bad = large.clone()
    bad[8:, ::7] = float("nan")               # tokens of a request that went wrong
    used.step(bad, [24, 24], tree)
    used.block.ws.fill_(255)                  # (scratch memory holds anything: NaN)
    used.seqs.step(ints([-24, -24]), 1)
    used.block.status.zero_()
    for more in ([5, 3], [1, 1]):
        got, want = (r.step(x, more, tree) for r in (used, fresh))
        n = sum(more)
        assert int(used.block.status.item()) == int(fresh.block.status.item()) == 0
        assert torch.equal(got[:n], want[:n]), more
        assert bool(torch.isfinite(got).all()) and torch.equal(got, want), more
        for r in (used, fresh):
            r.seqs.step(ints([-m for m in more]), 1)
