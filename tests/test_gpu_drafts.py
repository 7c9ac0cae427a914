"""The plan of a step, the masks of drafted trees and the move of an accepted path, each against a loop over its definition."""
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


def ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device=DEV)


# ---- the plan
def planned(lens, change, page, table, stack, count, prefix, T):
    """What the header says, in loops."""
    pages_of = lambda n: -(-n // page)
    table, stack = [list(r) for r in table], list(stack)
    returned = [table[b][j] for b, (n, c) in enumerate(zip(lens, change)) for j in range(pages_of(n + c), pages_of(n))]
    wanted = [(b, j) for b, (n, c) in enumerate(zip(lens, change)) for j in range(pages_of(n), pages_of(n + c))]
    for i, (b, j) in enumerate(wanted):
        table[b][j] = returned[i] if i < len(returned) else stack[count - 1 - (i - len(returned))]
    for i, p in enumerate(returned[len(wanted):]):
        stack[count + i] = p
    starts, pos, slot = [0], [], []
    for b, (n, c) in enumerate(zip(lens, change)):
        for i in range(max(c, 0)):
            pos.append(prefix + n + i)
            slot.append(table[b][(n + i) // page] * page + (n + i) % page)
        starts.append(len(pos))
    fill = T - len(pos)
    return ([n + c for n, c in zip(lens, change)], count + len(returned) - len(wanted), starts, pos + [0] * fill, slot + [-1] * fill, table, stack)


class Step:
    def __init__(self, lens, change, page=16, prefix=0, spare=7, extra_rows=0, width=None, seed=1, pages=None):
        g = torch.Generator()
        g.manual_seed(seed)
        used = [-(-n // page) for n in lens]
        after = [-(-max(0, n + c) // page) for n, c in zip(lens, change)]
        self.width = width or max(1, max(used + after))
        self.pages = max(1, pages or sum(used) + max(0, sum(after) - sum(used)) + spare)   # (a cache has a page)
        order = torch.randperm(self.pages, generator=g).tolist()
        self.table = [[-5] * (self.width + 2) for _ in lens]
        at = 0
        for b, n in enumerate(used):
            self.table[b][:n] = order[at:at + n]
            at += n
        self.count = self.pages - at
        self.stack = order[at:] + [-9] * at
        self.T = max(1, sum(max(0, c) for c in change) + extra_rows)
        self.lens, self.change, self.page, self.prefix = lens, change, page, prefix

    def run(self, B, T=None, stream=None):
        n, T = len(self.lens), T or self.T
        d = dict(table=ints(self.table), stack=ints(self.stack), lens=ints(self.lens), change=ints(self.change), count=ints([self.count]))
        out = dict(lens=torch.full((n,), -7, dtype=torch.int32, device=DEV), count=ints([-7]), starts=torch.full((n + 1,), -7, dtype=torch.int32, device=DEV),
                   pos=torch.full((T,), -7, dtype=torch.int32, device=DEV), slot=torch.full((T,), -7, dtype=torch.int64, device=DEV))
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        B.aweq_step_plan(d["lens"], d["change"], n, self.page, self.pages, d["table"], self.width + 2, self.width, d["stack"], d["count"], self.prefix, T, out["lens"],
                         out["count"], out["starts"], out["pos"], out["slot"], status, stream)
        got = (out["lens"].tolist(), int(out["count"]), out["starts"].tolist(), out["pos"].tolist(), out["slot"].tolist(), d["table"].tolist(), d["stack"].tolist())
        assert d["lens"].tolist() == self.lens and d["change"].tolist() == self.change and int(d["count"]) == self.count
        return got, int(status.item())

    def check(self, B, T=None):
        got, status = self.run(B, T)
        assert status == 0
        assert got == planned(self.lens, self.change, self.page, self.table, self.stack, self.count, self.prefix, T or self.T)

    def unchanged(self, B, T=None):
        """A step that is refused on the device; returns the status."""
        T = T or self.T
        got, status = self.run(B, T)
        assert got == (self.lens, self.count, [0] * (len(self.lens) + 1), [0] * T, [-1] * T, self.table, self.stack)
        return status


PLANS = {
    "one": ([0], [1]), "one_more": ([15], [1]), "next_page": ([16], [1]), "nothing": ([5], [0]), "all_goes": ([40], [-40]), "none": ([0], [0]),
    "prompts": ([0, 0, 0], [33, 1, 160]), "drafts": ([5, 16, 31, 32, 100], [4, 1, 17, 16, 7]), "rejected": ([20, 33, 64, 48], [-3, -1, -16, -17]),
    "more_given_than_taken": ([100, 3, 200, 17], [-90, 20, -200, 0]), "more_taken_than_given": ([100, 3, 0, 17], [-20, 90, 200, 1]),
}


@pytest.mark.parametrize("which", list(PLANS))
@pytest.mark.parametrize("page", [16, 64, 256])
def test_plan(B, which, page):
    lens, change = PLANS[which]
    for prefix, extra in ((0, 0), (1000, 5)):
        Step(lens, change, page, prefix, extra_rows=extra).check(B)
    Step(lens, change, page, spare=0).check(B)          # not a page too many


@pytest.mark.parametrize("n", [2, 63, 64, 65, 511, 512, 513, 1500, 8192])
def test_plan_of_many_sequences(B, n):
    lens = [(i * 7919) % 300 for i in range(n)]
    change = [((i * 31) % 23) - 5 if lens[i] > 20 else (i * 3) % 7 for i in range(n)]
    Step(lens, change, 16, 77, extra_rows=3, seed=n).check(B)
    Step(lens, [-v for v in lens], 32).check(B)


def test_plan_of_long_prompts(B):
    Step([0, 70000, 5], [50000, -65000, 30001], 64, 9, extra_rows=1).check(B)
    Step([0, 10], [20000, 1], 16).check(B)


def test_plans_that_are_refused_change_nothing(B):
    s = Step([10, 20, 30], [40, 5, 100], 16, spare=0)
    s.check(B)
    s.count -= 1
    s.stack = s.stack[:s.count] + [-9] * (s.pages - s.count)
    assert s.unchanged(B) == B.ST_PAGES
    assert Step([10, 20, 30], [4, 5, 6], extra_rows=2).unchanged(B, T=14) == B.ST_INDEX      # more tokens than rows
    assert Step([10, 20], [1, -21]).unchanged(B) == B.ST_INDEX                                # more taken away than there is
    assert Step([10, 20], [1, 30], width=3).unchanged(B) == B.ST_INDEX                        # longer than its row of pages
    s = Step([10, 20], [1, 1])
    s.lens = [10, -1]
    assert s.unchanged(B) == B.ST_INDEX
    s = Step([10, 20], [1, 2 ** 31 - 1], width=3, pages=20)
    s.T = 4
    assert s.unchanged(B) == B.ST_INDEX
    s = Step([40], [-40], spare=3)
    s.count = s.pages - 1          # a stack that would run over
    s.stack = list(range(s.pages))
    assert s.unchanged(B) == B.ST_INDEX
    s.count = -1
    assert s.unchanged(B) == B.ST_INDEX
    s = Step([128, 0], [-128, 128], width=8)
    s.pages = 4                    # a sequence that says it has more pages than there are
    s.count = 0
    assert s.unchanged(B) == B.ST_INDEX


# ---- masks
def family(parent):
    """Of each token, those on its path, itself among them."""
    seen = []
    for i, p in enumerate(parent):
        seen.append(({i} | seen[p]) if p >= 0 else {i})
    return seen


def words(seen, n):
    out = [sum(1 << j for j in seen if j // 64 == w) >> (64 * w) for w in range(n)]
    return [v - (1 << 64) if v >> 63 else v for v in out]


def tree(m, kind, seed=0):
    g = torch.Generator()
    g.manual_seed(seed + m)
    if kind == "chain":
        return list(range(-1, m - 1))
    if kind == "roots":
        return [-1] * m
    return [-1 if i == 0 or float(torch.rand(1, generator=g)) < 0.1 else int(torch.randint(0, i, (1,), generator=g)) for i in range(m)]


@pytest.mark.parametrize("kind", ["chain", "roots", "random"])
@pytest.mark.parametrize("new", [[1], [63], [64], [65, 0, 1], [5, 128, 17, 129], [1000, 3]])
def test_tree_mask(B, new, kind):
    T, prefix = sum(new), 50
    trees = [tree(m, kind, b) for b, m in enumerate(new)]
    lens = [m + 11 * b for b, m in enumerate(new)]
    need = -(-max(new) // 64)
    for ld, bound in ((need, max(new)), (need + 1, 64 * need)):
        mask = torch.full((T + 2, ld), 0x55, dtype=torch.int64, device=DEV)
        pos = torch.full((T + 2,), -3, dtype=torch.int32, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        starts = ints([sum(new[:b]) for b in range(len(new) + 1)])
        parent = ints([p for t in trees for p in t] + [0, 0])
        B.aweq_tree_mask(parent, T + 2, starts, len(new), bound, ints(lens), prefix, mask, ld, pos, status)
        want_mask, want_pos = [], []
        for b, t in enumerate(trees):
            for s in family(t):
                want_mask.append(words(s, need))
                want_pos.append(prefix + lens[b] - new[b] + len(s) - 1)
        assert int(status.item()) == 0
        assert mask[:T, :need].tolist() == want_mask and pos[:T].tolist() == want_pos
        assert (mask[T:] == 0x55).all() and (mask[:, need:] == 0x55).all() and (pos[T:] == -3).all()
        again = torch.zeros_like(mask)
        B.aweq_tree_mask(parent, T + 2, starts, len(new), bound, None, 0, again, ld, None, status)
        assert torch.equal(again[:T, :need], mask[:T, :need])


def test_parents_that_are_none(B):
    """Taken as the tree's beginning, and told of."""
    for wrong in (2, 7, -2, 2 ** 31 - 1, -2 ** 31):
        parent = [-1, 0, wrong, 2]
        mask, status = torch.zeros(4, 1, dtype=torch.int64, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        B.aweq_tree_mask(ints(parent), 4, ints([0, 4]), 1, 4, None, 0, mask, 1, None, status)
        assert int(status.item()) == B.ST_INDEX and mask.flatten().tolist() == [1, 3, 4, 12]
    for starts in ([0, 5], [-1, 4], [3, 2], [0, 9]):
        mask = torch.zeros(8, 1, dtype=torch.int64, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        B.aweq_tree_mask(ints([-1] * 8), 8, ints(starts), 1, 4, None, 0, mask, 1, None, status)
        assert int(status.item()) == B.ST_INDEX


# ---- the accepted path
class Path:
    def __init__(self, B, lens, new, kept, D=64, Hk=2, page=16, cache="f16", ld_extra=1, seed=1):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.lens, self.new, self.kept, self.D, self.Hk, self.page, self.cache = lens, new, kept, D, Hk, page, cache
        need = [-(-n // page) for n in lens]
        self.pages = sum(need) + 2
        order = torch.randperm(self.pages, generator=g, device=DEV).tolist()
        self.width = max(1, max(need))
        self.table = [[order[sum(need[:b]) + j] if j < need[b] else 10 ** 6 for j in range(self.width)] for b in range(len(lens))]
        dt = {"f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8}[cache]
        new_cache = lambda: torch.randint(-100, 100, (self.pages, Hk, page, D), generator=g, device=DEV).to(dt)
        self.caches = [new_cache(), new_cache()]
        self.steps = [torch.rand(self.pages, Hk, page, generator=g, device=DEV) for _ in range(2)] if cache == "i8" else [None, None]
        self.ld = max([1] + [len(k) for k in kept]) + ld_extra

    def run(self, B, count=None):
        n = len(self.lens)
        kept = ints([k + [77] * (self.ld - len(k)) for k in self.kept])
        change = torch.full((n,), 99, dtype=torch.int32, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        caches = [c.clone() for c in self.caches]
        steps = [None if s is None else s.clone() for s in self.steps]
        B.aweq_kv_keep(*caches, *steps, {"f16": B.AWEQ_F16, "bf16": B.AWEQ_BF16, "i8": B.AWEQ_I8}[self.cache], self.pages, self.page, self.Hk, self.D, ints(self.table),
                       self.width, ints(self.lens), ints([sum(self.new[:b]) for b in range(n + 1)]), n, max(1, sum(self.new)), kept, self.ld,
                       ints(count or [len(k) for k in self.kept]), change, status)
        return caches, steps, change.tolist(), int(status.item())

    def check(self, B, left=()):
        """left: sequences of which nothing is moved."""
        caches, steps, change, status = self.run(B)
        for before, after in zip(self.caches + self.steps, caches + steps):
            if before is None:
                continue
            want = before.clone()
            for b, (n, m, kept) in enumerate(zip(self.lens, self.new, self.kept)):
                if b in left:
                    continue
                at = lambda i: (self.table[b][i // self.page], i % self.page)
                for j, k in enumerate(kept):
                    (p, r), (s, t) = at(n - m + j), at(n - m + k)
                    want[p, :, r] = before[s, :, t]
            assert torch.equal(want.view(torch.uint8), after.view(torch.uint8))
        assert change == [0 if b in left else len(k) - m for b, (m, k) in enumerate(zip(self.new, self.kept))]
        return status


@pytest.mark.parametrize("cache", ["f16", "bf16", "i8"])
@pytest.mark.parametrize("D,Hk,page", [(64, 2, 16), (128, 3, 32), (256, 1, 64), (96, 2, 16), (8, 5, 16), (200, 1, 128)])
def test_kept_paths(B, cache, D, Hk, page):
    cases = [([7], [4], [[0, 2, 3]]), ([40, 5, 0, 16, 100], [12, 5, 0, 3, 64], [[3, 4, 5, 9], [], [], [2], [0, 1, 5, 6, 7, 20, 40, 63]]),
             ([300], [290], [list(range(1, 290))]), ([300, 290], [290, 290], [list(range(0, 290, 2)), list(range(290))]), ([33] * 20, [17] * 20, [[b % 17] for b in range(20)])]
    for lens, new, kept in cases:
        assert Path(B, lens, new, kept, D, Hk, page, cache).check(B) == 0


def test_paths_that_are_refused(B):
    lens, new = [40, 30, 20], [12, 8, 5]
    for wrong in ([0, 2, 2], [3, 1], [0, 8], [-1, 2]):
        assert Path(B, lens, new, [[1, 5], wrong, [4]]).check(B, left=(1,)) == B.ST_INDEX
    for n in (-1, 9, 100):
        p = Path(B, lens, new, [[1, 5], [0, 1, 2, 3, 4, 5, 6, 7], [4]], ld_extra=3)
        caches, _, change, status = p.run(B, count=[2, n, 1])
        assert status == B.ST_INDEX and change[1] == 0 and change[0] == -10
    p = Path(B, lens, new, [[1, 5], [2], [4]])
    p.lens = [40, 7, 20]           # fewer than its new tokens
    assert p.check(B, left=(1,)) == B.ST_INDEX
    p = Path(B, lens, new, [[1, 5], [2], [4]])
    p.table[1][1] = p.pages        # a page that there is not
    caches, _, change, status = p.run(B)
    assert status == B.ST_INDEX
    p = Path(B, lens, new, [[1, 5], [2], [4]])
    p.lens = [40, 10 ** 6, 20]     # longer than the table's rows
    assert p.check(B, left=(1,)) == B.ST_INDEX
