"""Attention over values that are hard on a softmax, in every form that the sizes lead to: what is not finite, in queries, keys and steps, reaches the
tokens that see it, and nobody else, however the keys are split.  Against softmax in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
PAGE = 32


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2311_01305_amd import binding
    binding.load_library()
    return binding


# name: lens, new, prefix, Hq, Hk, and whether partial results are joined
FORMS = {
    "one_part": ([60, 7], [1, 1], 0, 4, 2, False),
    "parts": ([1500, 40], [1, 1], 0, 4, 2, True),
    "behind_a_prefix": ([30, 200, 5], [1, 1, 1], 700, 4, 2, True),
    "many_behind_a_prefix": ([9] * 40, [1] * 40, 700, 4, 2, True),
    "some_new": ([70, 40], [3, 4], 0, 4, 2, False),
    "some_new_parts": ([900, 40], [3, 4], 300, 4, 2, True),
    "prompts": ([300, 65], [300, 65], 0, 64, 32, False),
    "prompts_behind_a_prefix": ([150, 129], [150, 129], 500, 128, 64, False),
    "chunk": ([2000, 20], [20, 9], 300, 4, 2, True),
}


class Batch:
    """Queries [T, Hq, D], and keys and values [n, Hk, D] of the prefix and of each sequence, in the 64-bit values that the cache stands for; of codes
    also their steps.  A test changes them before put() lays them out."""

    def __init__(self, dt, codes, D, lens, new, prefix, Hq, Hk, seed=1):
        self.__dict__.update(dt=dt, codes=codes, D=D, lens=lens, new=new, prefix=prefix, Hq=Hq, Hk=Hk, scale=D ** -0.5, past=1.0)
        g = torch.Generator()
        g.manual_seed(seed)
        normal = lambda *s: torch.randn(s, generator=g)
        self.T = sum(new)
        self.q = (2 * normal(self.T, Hq, D)).to(TYPES[dt])
        self.k, self.v, self.ks, self.vs = [], [], [], []
        for n in [prefix] + lens:
            for c, s in ((self.k, self.ks), (self.v, self.vs)):
                x = normal(n, Hk, D)
                if codes:
                    step = x.abs().amax(2) / 127
                    c.append(torch.round(x / step[..., None]).to(torch.int8))
                    s.append(step)
                else:
                    c.append(x.to(TYPES[dt]))
                    s.append(None)

    def run(self, B, joined=None):
        D, Hk, Hq, T, n_seq = self.D, self.Hk, self.Hq, self.T, len(self.lens)
        need = [-(-n // PAGE) for n in [self.prefix] + self.lens]
        pages, width = sum(need) + 1, max(1, max(need[1:]))
        store = torch.int8 if self.codes else TYPES[self.dt]
        table = torch.full((n_seq, width), -1, dtype=torch.int32)
        at, places = 0, []
        for i, n in enumerate(need):
            places.append(torch.arange(at, at + n))
            if i:
                table[i - 1, :n] = places[-1]
            at += n
        cache, steps = [], []
        for c, s in ((self.k, self.ks), (self.v, self.vs)):
            whole, whole_s = torch.zeros(pages, Hk, PAGE, D, dtype=store), torch.full((pages, Hk, PAGE), self.past)
            for x, xs, p in zip(c, s, places):
                r = torch.arange(x.shape[0])
                whole[p[r // PAGE], :, r % PAGE] = x
                if self.codes:
                    whole_s[p[r // PAGE], :, r % PAGE] = xs
            cache.append(whole.to(DEV))
            steps.append(whole_s.to(DEV) if self.codes else None)
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
        code = {"f16": B.AWEQ_F16, "bf16": B.AWEQ_BF16}[self.dt]
        out, lse = torch.full((T, Hq * D), 4.0, dtype=TYPES[self.dt], device=DEV), torch.full((T, Hq), 7.0, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        most, tokens = max(self.lens), max(self.new)
        size = B.aweq_prefix_attention_ws(T, Hq, Hk, D, n_seq, tokens, self.prefix, most)
        assert joined is None or (size > 0) == joined
        ws = torch.full((size // 4 + 4,), float("nan"), device=DEV)
        B.aweq_prefix_attention(self.q.to(DEV), code, T, Hq, D, Hq * D, cache[0], cache[1], steps[0], steps[1], B.AWEQ_I8 if self.codes else code, pages, PAGE, Hk,
                                places[0].to(torch.int32).to(DEV) if need[0] else None, self.prefix, table.to(DEV), width, ints(self.lens),
                                ints([sum(self.new[:b]) for b in range(n_seq + 1)]), n_seq, most, tokens, self.scale, out, Hq * D, lse, ws, status, ws_bytes=size)
        assert int(status.item()) == 0
        return out.double().cpu().view(T, Hk, Hq // Hk, D), lse.double().cpu().view(T, Hk, Hq // Hk)

    def values(self, which):
        c, s = ((self.k, self.ks), (self.v, self.vs))[which]
        return [x.double() * (xs.double()[..., None] if self.codes else 1.0) for x, xs in zip(c, s)]

    def check(self, out, lse, exact_scores=False):
        """Finite where the definition is, and near it: the probabilities' and the output's rounding, 2e-5 and 2^-21 of the products' sizes for scores,
        exponentials and sums; probabilities in binary16 are no finer than 2^-25 of the largest, the outputs no finer than their type."""
        floor = 2.0 ** -24 if self.dt == "f16" else 2.0 ** -130
        D = self.D
        heads = sorted({0, min(1, self.Hk - 1), self.Hk - 1})      # (of the keys; what is planted is in the first)
        out, lse, q = out[:, heads], lse[:, heads], self.q.double().view(self.T, self.Hk, -1, D)[:, heads]
        k, v = ([x[:, heads] for x in self.values(i)] for i in range(2))
        unit = 2.0 ** -11 if self.dt == "f16" else 2.0 ** -8
        p_unit = 2.0 ** -11 if self.codes else unit
        t = 0
        for b, (n, m) in enumerate(zip(self.lens, self.new)):
            for i in range(m):
                own, t = max(0, n - m + 1 + i), t + 1
                if m > 20 and i % 13 and abs(own - 1 - n // 2) > 2:     # (of a prompt some, and those next to what is planted)
                    continue
                keys, vals = (torch.cat((x[0], x[1 + b][:own])).transpose(0, 1) for x in (k, v))     # [Hk, seen, D]
                got, l = out[t - 1], lse[t - 1]
                s = (q[t - 1] @ keys.transpose(1, 2)) * self.scale
                where = (b, i, self.dt, self.codes, D)
                top = s.amax(2, keepdim=True) if s.shape[2] else torch.full(s.shape[:2] + (1,), -math.inf, dtype=s.dtype)
                e = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
                total = e.sum(2, keepdim=True)
                none = total == 0
                want = torch.where(none, torch.zeros_like(total), (e @ vals) / torch.where(none, torch.ones_like(total), total))
                exact = torch.where(none, torch.full_like(top, -math.inf), top + torch.log(total))[..., 0]
                assert torch.equal(torch.isfinite(got), torch.isfinite(want)), where
                assert torch.equal(torch.isnan(l), torch.isnan(exact)) and torch.equal(l == -math.inf, exact == -math.inf), where
                clean = lambda x: torch.nan_to_num(x.abs(), 0.0, 0.0, 0.0)
                sizes = (clean(q[t - 1]) @ clean(keys).transpose(1, 2)).amax(2) * self.scale if s.shape[2] else torch.zeros(s.shape[:2], dtype=s.dtype)
                if exact_scores:
                    sizes = torch.zeros_like(sizes)
                around = torch.nan_to_num(e, 0.0) @ clean(vals) / torch.nan_to_num(total, 1.0).clamp(min=1e-300)
                biggest = clean(vals).amax() if s.shape[2] else 0.0
                small = 2.0 ** -25 * s.shape[2] * biggest / total.clamp(min=1.0) if p_unit == 2.0 ** -11 else 0.0
                allowed = (1.01 * p_unit + 2e-5 + 2.0 ** -21 * sizes[..., None]) * around + 1.01 * unit * want.abs() + small + floor
                off = (got - want).abs()
                ok = torch.isfinite(want)
                assert (off <= allowed)[ok].all(), (where, float((off - allowed)[ok].max()))
                fine = torch.isfinite(exact)
                assert ((l - exact).abs() <= 1e-5 + 2.0 ** -21 * sizes + 2.0 ** -22 * exact.abs())[fine].all(), where


KINDS = [("f16", False), ("bf16", False), ("f16", True), ("bf16", True)]


def somewhere(b):
    """(range, key) of a key in the prefix, if there is one, and in the middle of the first sequence: its later tokens alone see that one."""
    return ([(0, b.prefix // 3)] if b.prefix else []) + [(1, b.lens[0] // 2)]


@pytest.mark.parametrize("dt,codes", KINDS)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("form", list(FORMS))
def test_scores_that_are_not_finite(B, form, D, dt, codes):
    lens, new, prefix, Hq, Hk, joined = FORMS[form]
    for plant in ("nothing", "nan_key", "inf_key", "nan_query", "inf_query"):
        if plant == "inf_key" and codes:
            continue      # (a step is finite or NaN)
        print(f"[values] {form} D={D} {dt} codes={codes} {plant}", flush=True)
        base = Batch(dt, codes, D, lens, new, prefix, Hq, Hk, seed=D)
        for r, j in somewhere(base) if plant.endswith("key") else [(1, 0)]:
            b = Batch(dt, codes, D, lens, new, prefix, Hq, Hk, seed=D)
            if plant == "nan_key" and codes:
                b.ks[r][j, 0] = float("nan")
            elif plant.endswith("key"):
                b.k[r][j, 0, 3] = float(plant[:3])
            elif plant.endswith("query"):
                b.q[b.T // 2, 1, 5] = float(plant[:3])
            b.check(*b.run(B, joined))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", list(FORMS))
def test_a_score_of_minus_infinity_leaves_its_key_out(B, form, D):
    """In some keys, and in all that a token sees: no key at all, then."""
    lens, new, prefix, Hq, Hk, joined = FORMS[form]
    for every in (False, True):
        b = Batch("f16", False, D, lens, new, prefix, Hq, Hk, seed=D)
        b.q[..., 3] = b.q[..., 3].abs() + 0.5
        for r, j in somewhere(b):
            b.k[r][j, 0, 3] = -math.inf
        if every:
            for x in b.k:
                x[:, 0, 3] = -math.inf
        out, lse = b.run(B, joined)
        b.check(out, lse)
        if every:
            assert (out[:, 0] == 0).all() and (lse[:, 0] == -math.inf).all()


def large_scores(B, form, dt, codes):
    """Scores of 2^30 and more that are whole numbers of a power of two, so that their sums are exact and the largest ones often equal."""
    lens, new, prefix, Hq, Hk, joined = FORMS[form]
    for D in (64, 128):
        b = Batch(dt, codes, D, lens, new, prefix, Hq, Hk, seed=D)
        g = torch.Generator()
        g.manual_seed(D)
        whole = lambda x: torch.randint(-3, 4, x.shape, generator=g)
        b.q = (whole(b.q) * 2.0 ** (13 if dt == "f16" else 50)).to(TYPES[dt])
        for r, x in enumerate(b.k):
            b.k[r] = whole(x).to(torch.int8) if codes else (whole(x) * 2.0 ** (13 if dt == "f16" else 50)).to(TYPES[dt])
            if codes:
                b.ks[r].fill_(2.0 ** 20)
        b.scale = 0.25
        print(f"[values] {form} D={D} {dt} codes={codes} large scores", flush=True)
        out, lse = b.run(B, joined)
        b.check(out, lse, exact_scores=True)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("form", list(FORMS))
def test_scores_of_any_size(B, form, dt):
    large_scores(B, form, dt, False)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("form", list(FORMS))
def test_steps_of_any_size(B, form, D, dt):
    """A value's step says nothing about its key's weight: the smallest normal number in all keys or in a few of them, sizes spread over many orders, and
    large ones in keys that earlier tokens do not see."""
    lens, new, prefix, Hq, Hk, joined = FORMS[form]
    tiny = 2.0 ** -126
    spread = (-30, 6) if dt == "f16" else (-80, 30)
    for kind in ("all_tiny", "five_tiny", "every_other_tiny", "spread", "large_last"):
        print(f"[values] {form} D={D} {dt} steps: {kind}", flush=True)
        b = Batch(dt, True, D, lens, new, prefix, Hq, Hk, seed=D)
        g = torch.Generator()
        g.manual_seed(D)
        for r, s in enumerate(b.vs):
            n = s.shape[0]
            if kind == "all_tiny":
                s.fill_(tiny)
            elif kind == "five_tiny":
                s[torch.randperm(n, generator=g)[:5]] = tiny
            elif kind == "every_other_tiny":
                s[::2] = tiny
            elif kind == "spread":
                s *= 2.0 ** torch.randint(*spread, s.shape, generator=g)
            elif r and n > 1:
                s[-(-n // 2):] *= 2.0 ** spread[1]
        b.check(*b.run(B, joined))


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("form", list(FORMS))
def test_scores_of_any_size_over_codes(B, form, dt):
    large_scores(B, form, dt, True)


@pytest.mark.parametrize("dt,codes", KINDS)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("form", list(FORMS))
def test_values_that_are_not_finite(B, form, D, dt, codes):
    """They reach the tokens that see their key; the same sequence's earlier tokens, whose probability of it is 0, have none of it."""
    lens, new, prefix, Hq, Hk, joined = FORMS[form]
    for plant in ("nan",) if codes else ("nan", "inf", "-inf"):
        print(f"[values] {form} D={D} {dt} codes={codes} {plant} in a value", flush=True)
        base = Batch(dt, codes, D, lens, new, prefix, Hq, Hk, seed=D)
        for r, j in somewhere(base) + [(1, lens[0] - 1)]:
            b = Batch(dt, codes, D, lens, new, prefix, Hq, Hk, seed=D)
            if codes:
                b.vs[r][j, 0] = float(plant)
            else:
                b.v[r][j, 0, 7] = float(plant)
            b.check(*b.run(B, joined))


@pytest.mark.parametrize("form", list(FORMS))
def test_small_steps_before_any_others(B, form):
    """The smallest steps, and behind the last key of each page whatever a page may hold."""
    lens, new, prefix, Hq, Hk, joined = FORMS[form]
    for D in (64, 128, 256):
        for past in (2.0 ** 100, float("inf"), float("nan"), 0.0):
            print(f"[values] {form} D={D} small steps before {past}", flush=True)
            b = Batch("bf16", True, D, lens, new, prefix, Hq, Hk, seed=D)
            b.past = past
            for s in b.vs:
                s.fill_(2.0 ** -126)
            b.check(*b.run(B, joined))
