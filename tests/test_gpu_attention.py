"""Attention over a shared prefix and each sequence's own pages against softmax in 64 bits, one sequence after the other."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2311_01305_amd import binding
    binding.load_library()
    return binding


def dt_of(B, name):
    return {"f16": B.AWEQ_F16, "bf16": B.AWEQ_BF16, "i8": B.AWEQ_I8}[name]


class Case:
    """A batch: lens own keys and new tokens of each sequence, prefix tokens shared; pages in any order, everything that is no key left as NaN."""

    def __init__(self, dt, cache, D, Hq, Hk, page, lens, new, prefix, seed=1, ld_extra=0, spare=2, loud=1.0, one_each=False):
        self.__dict__.update(dt=dt, cache=cache, D=D, Hq=Hq, Hk=Hk, page=page, lens=lens, new=new, prefix=prefix, one_each=one_each)
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        normal = lambda *s: torch.randn(s, generator=g, device=DEV)
        need = [-(-n // page) for n in lens]
        pp = -(-prefix // page)
        self.pages = pp + sum(need) + spare
        order = torch.randperm(self.pages, generator=g, device=DEV).to(torch.int32)
        self.prefix_table = order[:pp].contiguous()
        self.width = max(1, max(need)) + 1
        self.table = torch.full((len(lens), self.width), -1, dtype=torch.int32, device=DEV)
        at = pp
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.T = sum(new)
        self.ldq = Hq * D + ld_extra
        self.q = torch.full((self.T, self.ldq), float("nan"), dtype=TYPES[dt], device=DEV)
        self.q[:, :Hq * D] = (normal(self.T, Hq * D) * 2 * loud).to(TYPES[dt])
        store = torch.int8 if cache == "i8" else TYPES[dt]
        self.k, self.v = (torch.full((self.pages, Hk, page, D), 99 if cache == "i8" else float("nan"), dtype=store, device=DEV) for _ in range(2))
        self.ks, self.vs = (torch.full((self.pages, Hk, page), float("nan"), device=DEV) for _ in range(2)) if cache == "i8" else (None, None)
        ranges = [(self.prefix_table, prefix)] + [(self.table[b], n) for b, n in enumerate(lens)]
        self.keys = []
        for table, n in ranges:
            both = []
            for c, s, size in ((self.k, self.ks, 1.0), (self.v, self.vs, 3.0)):
                x = normal(n, Hk, D) * size
                p, r = table[torch.arange(n, device=DEV) // page].long(), torch.arange(n, device=DEV) % page
                if cache == "i8":
                    x *= torch.exp(normal(n, Hk, 1))      # steps that differ from token to token
                    step = x.abs().amax(2) / 127
                    x = torch.round(x / step[..., None])
                    s[p, :, r] = step
                    both.append(x.double() * step.double()[..., None])
                    c[p, :, r] = x.to(torch.int8)
                else:
                    x = x.to(store)
                    both.append(x.double())
                    c[p, :, r] = x
            self.keys.append([x.transpose(0, 1).cpu() for x in both])    # [Hk, n, D]
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
        self.lens_d = ints(lens)
        self.q_start = None if one_each else ints([sum(new[:b]) for b in range(len(lens) + 1)])
        self.scale = 1 / math.sqrt(D)
        self.max_len, self.max_q = max(lens), max(new)

    def run(self, B, out=None, max_len=None, max_q=None, stream=None):
        ldo = self.Hq * self.D + 8
        out = torch.full((self.T, ldo), 4.0, dtype=TYPES[self.dt], device=DEV) if out is None else out
        lse = torch.full((self.T, self.Hq), 7.0, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        max_len, max_q = max_len or self.max_len, max_q or self.max_q
        n = B.aweq_prefix_attention_ws(self.T, self.Hq, self.Hk, self.D, len(self.lens), max_q, self.prefix, max_len)
        ws = torch.full((n // 4 + 4,), float("nan"), device=DEV)
        B.aweq_prefix_attention(self.q, dt_of(B, self.dt), self.T, self.Hq, self.D, self.ldq, self.k, self.v, self.ks, self.vs,
                                dt_of(B, self.cache if self.cache == "i8" else self.dt), self.pages, self.page, self.Hk, self.prefix_table, self.prefix,
                                self.table, self.width, self.lens_d, self.q_start, len(self.lens), max_len, max_q, self.scale, out, ldo, lse,
                                ws if n else None, status, stream, ws_bytes=n)
        assert (out[:, self.Hq * self.D:] == 4.0).all()
        return out[:, :self.Hq * self.D], lse, int(status.item())

    def check(self, out, lse):
        """Within: the probabilities' rounding for the product with v (relative 2^-11 or 2^-8 each; binary16 ones are no finer than 2^-25 of the
        largest), the output's own, and 2e-5 for scores (sums of D products in fp32 of |scores| up to some ten), exponentials and sums."""
        G, D = self.Hq // self.Hk, self.D
        q = self.q[:, :self.Hq * D].double().cpu().view(self.T, self.Hk, G, D)
        got, lse = out.double().cpu().view(self.T, self.Hk, G, D), lse.double().cpu().view(self.T, self.Hk, G)
        unit = 2.0 ** -11 if self.dt == "f16" else 2.0 ** -8
        p_unit = unit if self.cache != "i8" else 2.0 ** -11
        t = 0
        for b, (n, m) in enumerate(zip(self.lens, self.new)):
            k, v = (torch.cat((self.keys[0][i], self.keys[1 + b][i]), 1) for i in range(2))
            for i in range(m):
                seen = self.prefix + max(0, n - m + 1 + i if n >= m or m > 1 else 0)
                seen = min(seen, self.prefix + n)
                o, l = got[t], lse[t]
                t += 1
                if seen == 0:
                    assert (o == 0).all() and (l == -math.inf).all()
                    continue
                s = torch.matmul(q[t - 1], k[:, :seen].transpose(1, 2)) * self.scale          # [Hk, G, seen]
                sizes = torch.matmul(q[t - 1].abs(), k[:, :seen].abs().transpose(1, 2)).amax(2) * self.scale
                top = s.amax(2, keepdim=True)
                e = torch.exp(s - top)
                total = e.sum(2, keepdim=True)
                want = torch.matmul(e, v[:, :seen]) / total
                around = torch.matmul(e, v[:, :seen].abs()) / total
                score = 2e-5 + 2.0 ** -21 * sizes[..., None]
                small = 2.0 ** -25 * seen * v[:, :seen].abs().amax() / total if p_unit == 2.0 ** -11 else 0.0
                allowed = 1.01 * p_unit * around + 1.01 * unit * want.abs() + score * around + small + 2.0 ** -24
                off = (o - want).abs()
                assert (off <= allowed).all(), (b, i, float(off.max()), float((off / allowed).max()))
                exact = (top + torch.log(total))[..., 0]
                assert ((l - exact).abs() <= 1e-5 + 2.0 ** -21 * sizes + 2.0 ** -22 * exact.abs()).all(), (b, i, (l - exact).abs().max())

    def all(self, B, **k):
        out, lse, status = self.run(B, **k)
        assert status == 0
        self.check(out, lse)


LENS = {
    "one": ([1], [1]),
    "nothing": ([0, 0], [1, 1]),
    "some_empty": ([0, 5, 0, 33, 16], [1, 1, 1, 1, 1]),
    "ragged": ([1, 15, 16, 17, 31, 32, 33, 64, 100, 129], [1] * 10),
    "long": ([1500, 3, 2049], [1, 1, 1]),
    "prompts": ([40, 1, 130, 64], [40, 1, 130, 64]),
    "chunks": ([200, 7, 64, 300], [3, 7, 17, 40]),
    "cut": ([2, 9], [5, 4]),                       # the first tokens see no key of their own
    "none_new": ([50, 20, 8], [4, 0, 2]),
}


@pytest.mark.parametrize("cache", ["f16", "bf16", "f16_i8", "bf16_i8"])
@pytest.mark.parametrize("D,Hq,Hk,page", [(128, 8, 2, 16), (64, 3, 3, 64), (256, 4, 1, 32), (128, 32, 1, 128)])
@pytest.mark.parametrize("which", list(LENS))
def test_own_keys_and_prefix(B, which, D, Hq, Hk, page, cache):
    lens, new = LENS[which]
    dt = cache.split("_")[0]
    for prefix in (0, 1, 77, 640):
        print(f"[attention] {which} D={D} Hq={Hq} Hk={Hk} page={page} {cache} prefix={prefix}", flush=True)
        Case(dt, "i8" if cache.endswith("i8") else "same", D, Hq, Hk, page, lens, new, prefix, seed=prefix + D, ld_extra=8 * (prefix % 2)).all(B)


@pytest.mark.parametrize("cache", ["same", "i8"])
def test_one_token_each_without_starts(B, cache):
    Case("f16", cache, 128, 8, 8, 16, [3, 0, 70, 18], [1, 1, 1, 1], 33, one_each=True).all(B)
    Case("bf16", cache, 64, 8, 4, 32, [300], [1], 0, one_each=True).all(B)


def test_many_rows_against_the_prefix(B):
    """Rows of the batch fill tiles of 64 and 128, with and without a remainder."""
    for B_, G in ((4, 4), (17, 4), (64, 1), (65, 1), (70, 2), (33, 8)):
        lens = [(7 * i) % 40 for i in range(B_)]
        print(f"[attention] batch {B_} x {G}", flush=True)
        Case("f16", "same", 128, 2 * G, 2, 16, lens, [1] * B_, 1000, seed=B_).all(B)
        Case("bf16", "i8", 128, 2 * G, 2, 16, lens, [1] * B_, 700, seed=B_).all(B)


def test_sharp_and_flat_scores(B):
    """Scores that differ by hundreds (one key takes all) and by nothing."""
    for loud in (0.0, 30.0):
        for cache in ("same", "i8"):
            Case("f16", cache, 128, 8, 2, 32, [500, 41], [1, 1], 300, seed=3, loud=loud).all(B)


def test_bounds_larger_than_the_batch(B):
    """max_len and max_q are bounds: larger ones lay the launch out otherwise and change nothing else."""
    c = Case("f16", "same", 128, 8, 2, 16, [90, 5, 33], [4, 1, 2], 50, seed=9)
    c.all(B, max_len=5000, max_q=7)


def test_out_of_range_pages_and_lengths_are_reported(B):
    c = Case("f16", "same", 128, 8, 2, 16, [40, 70], [1, 1], 20, seed=9)
    c.table[1, 2] = c.pages
    assert c.run(B)[2] == B.ST_INDEX
    c = Case("f16", "same", 128, 8, 2, 16, [40, 70], [1, 1], 20, seed=9)
    assert c.run(B, max_len=60)[2] == B.ST_INDEX           # a length over max_len
    c.lens_d[0] = -3
    assert c.run(B)[2] == B.ST_INDEX
    c.lens_d[0] = 40
    c.q_start[1] = 5
    assert c.run(B)[2] == B.ST_INDEX


def test_repeats_are_the_same_to_the_bit_and_streams(B):
    c = Case("f16", "same", 128, 8, 2, 16, [900, 5, 333], [1, 1, 1], 700, seed=2)
    a = c.run(B)
    b = c.run(B)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        d = c.run(B)
    side.synchronize()
    assert torch.equal(a[0], d[0]) and torch.equal(a[1], d[1])


def test_cache_past_32_bits(B):
    """Pages whose byte offset needs more than 32 bits."""
    Hk, D, page, pages, n = 8, 128, 256, 9000, 300
    k, v = (torch.full((pages, Hk, page, D), float("nan"), dtype=torch.float16, device=DEV) for _ in range(2))
    table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device=DEV)
    ks, vs = torch.randn(n, Hk, D, device=DEV).half(), torch.randn(n, Hk, D, device=DEV).half()
    at = torch.arange(n, device=DEV)
    for c, x in ((k, ks), (v, vs)):
        c[table[0, at // page].long(), :, at % page] = x
    q = torch.randn(1, Hk * D, device=DEV).half()
    out, lens = torch.empty_like(q), torch.tensor([n], dtype=torch.int32, device=DEV)
    size = B.aweq_prefix_attention_ws(1, Hk, Hk, D, 1, 1, 0, n)
    ws = torch.empty(max(16, size), dtype=torch.uint8, device=DEV)
    B.aweq_prefix_attention(q, B.AWEQ_F16, 1, Hk, D, Hk * D, k, v, None, None, B.AWEQ_F16, pages, page, Hk, None, 0, table, 2, lens, None, 1, n, 1, D ** -0.5, out,
                            Hk * D, None, ws)
    s = torch.einsum("hd,nhd->hn", q.view(Hk, D).double().cpu(), ks.double().cpu()) * D ** -0.5
    want = torch.einsum("hn,nhd->hd", torch.softmax(s, 1), vs.double().cpu()).flatten()
    assert np.abs(out[0].double().cpu() - want).max() <= 2.0 ** -10 * 4
