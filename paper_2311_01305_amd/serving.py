"""The attention block of a served decoder on the quantised layers that the calibration leaves: the projections as int8 products whose tokens
are quantised on the way, norm and rotation of the heads on the way into a paged cache, attention over the sequences' own pages and a prefix
that all of them share.  Four calls of the library for a step of any tokens, one of each sequence or whole prompts:

    aweq_w8a8_gemm_tokens (q, k, v)  ->  aweq_kv_append  ->  aweq_prefix_attention  ->  aweq_w8a8_gemm_tokens (output)

The projections may be 4-bit floating point instead (aweq_mx4_gemm_tokens), and the new tokens of a sequence a tree of drafts of which a path is kept
(aweq_tree_attention); Sequences plans such steps on the device:

    aweq_step_plan  ->  aweq_tree_mask  ->  the block's four calls  ->  aweq_kv_keep  ->  aweq_step_plan

`python -m paper_2311_01305_amd.serving` calibrates a block's projections on synthetic activations, runs a shared prompt once and decodes a batch
behind it (--draft: in trees of that many tokens; --mx4: 4-bit projections).  No arithmetic of the operators happens here.
"""
import argparse
import time
from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

from . import binding as B
from . import pipeline

DTYPES = {torch.float16: B.AWEQ_F16, torch.bfloat16: B.AWEQ_BF16}


@dataclass
class QuantLinear:
    """An 8-bit layer as pipeline.calibrate_layer leaves it, or several that read the same input as one.  inv_s: the equalization's 1 / s, or None where what
    produces the input has it folded in."""
    N: int
    K: int
    codes: torch.Tensor
    step_w: torch.Tensor
    zero_w: torch.Tensor
    rowsum_w: torch.Tensor
    bias: Optional[torch.Tensor] = None
    inv_s: Optional[torch.Tensor] = None
    w_group: int = 0

    @classmethod
    def from_layer(cls, buf: pipeline.LayerBuffers, fold: bool = True, bias: Optional[torch.Tensor] = None, correct: bool = True):
        """bias: the layer's own, before any correction.  correct: with the mean error that its weights' codes make on the calibration tokens taken off
        (Eq. 12-15).  (The calibration's bias_out has the mean error of its static activation quantizer in it as well, which is not the tokens' here.)"""
        t = buf.t
        if buf.bits != 8 or buf.group > 0:
            raise ValueError("8-bit weights with a scale for each output channel or the tensor")
        return cls(buf.N, buf.K, t["codes"], t["step_w"], t["zero_w"], t["rowsum_w"], _bias(t, t, buf.N, buf.K, buf.group, bias) if correct else bias,
                   t["inv_s"] if fold else None, buf.group)

    @classmethod
    def from_group(cls, gb: pipeline.GroupBuffers, fold: bool = True, biases: Optional[Sequence] = None, correct: bool = True):
        """The layers of pipeline.calibrate_group side by side as one, such as queries, keys and values; biases: of each, as in from_layer."""
        biases = [None] * len(gb.Ns) if biases is None else list(biases)
        if len(biases) != len(gb.Ns):
            raise ValueError("a bias, or None, for each layer")
        join = lambda name: torch.cat([p[name] for p in gb.per])
        codes = torch.cat([p["codes"].view(-1, N, 64) for p, N in zip(gb.per, gb.Ns)], 1).flatten()      # (panels of 64 inputs, the channels in each)
        if correct:
            biases = [_bias(gb.t, p, N, gb.K, 0, b) for p, N, b in zip(gb.per, gb.Ns, biases)]
        elif any(b is not None for b in biases):
            biases = [torch.zeros_like(p["step_w"]) if b is None else b for p, b in zip(gb.per, biases)]
        bias = None if biases[0] is None else torch.cat(biases)
        return cls(sum(gb.Ns), gb.K, codes, join("step_w"), join("zero_w"), join("rowsum_w"), bias, gb.t["inv_s"] if fold else None, 0)


@dataclass
class Mx4Linear:
    """A layer whose weight is in microscaled 4-bit floating point (aweq_quant_mx4), its tokens quantised the same way in the product.  factor: what the
    input's channels are multiplied by first (an equalization's 1 / s), or None.  bias: the layer's own, as it is: unlike a QuantLinear's it has no mean error of the
    codes taken off (Eq. 12-15 is of a quantizer whose errors the calibration has measured, which it does for integers alone)."""
    N: int
    K: int
    codes: torch.Tensor
    scales: torch.Tensor
    bias: Optional[torch.Tensor] = None
    factor: Optional[torch.Tensor] = None

    @classmethod
    def from_weight(cls, W: torch.Tensor, bias: Optional[torch.Tensor] = None, factor: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
        """W [N x K], float32, float16 or bfloat16, rows in one piece; N a multiple of 4, K of 32."""
        if W.dim() != 2 or W.stride(1) != 1:
            raise ValueError("a matrix whose rows are in one piece")
        N, K = W.shape
        if N % 4 or not B.aweq_mx4_code_bytes(N, K):
            raise ValueError("output channels in fours and input channels in blocks of 32, up to 2^20: the product reads no others")
        if factor is not None:
            _check("factor", factor, torch.float32, (K,), W.device)
        if bias is not None:
            _check("bias", bias, torch.float32, (N,), W.device)
        codes, scales = (torch.empty(n(N, K), dtype=torch.uint8, device=W.device) for n in (B.aweq_mx4_code_bytes, B.aweq_mx4_scale_bytes))
        B.aweq_quant_mx4(W, pipeline._dt(W) if W.dtype != torch.bfloat16 else B.AWEQ_BF16, N, K, W.stride(0), None, codes, scales, status)
        return cls(N, K, codes, scales, bias, factor)

    @classmethod
    def from_layer(cls, buf: pipeline.LayerBuffers, fold: bool = True, bias: Optional[torch.Tensor] = None):
        """The equalised weight of a layer that pipeline.calibrate_layer has been through; fold: with the equalization's 1 / s on its input."""
        t = buf.t
        return cls.from_weight(t["W_hat"], bias, t["inv_s"] if fold else None, t["status"])

    @classmethod
    def from_group(cls, gb: pipeline.GroupBuffers, fold: bool = True, biases: Optional[Sequence] = None):
        """The layers of pipeline.calibrate_group side by side as one; biases: of each, or None."""
        biases = [None] * len(gb.Ns) if biases is None else list(biases)
        if len(biases) != len(gb.Ns):
            raise ValueError("a bias, or None, for each layer")
        for i, (b, N) in enumerate(zip(biases, gb.Ns)):
            if b is not None:
                _check(f"bias {i}", b, torch.float32, (N,), gb.per[i]["W_hat"].device)
        bias = None
        if any(b is not None for b in biases):
            bias = torch.cat([torch.zeros_like(p["step_w"]) if b is None else b for p, b in zip(gb.per, biases)])
        return cls.from_weight(torch.cat([p["W_hat"] for p in gb.per]), bias, gb.t["inv_s"] if fold else None, gb.t["status"])


def _bias(t, layer, N, K, group, bias):
    """A bias less the mean output of what its layer's codes are off the folded weight by."""
    W = layer["W_hat"]
    delta, out = torch.empty_like(layer["bias_out"]), torch.empty_like(layer["bias_out"])
    B.aweq_bias_correct(B.BIAS_WEIGHT_ONLY, W, pipeline._dt(W), N, K, W.stride(0), t["mu_xhat"], 0, None, None, None, None, None, layer["codes"], 8, group,
                        layer["step_w"], layer["zero_w"], bias, delta, out, True, t["status"])
    return out


class PagedCache:
    """Pages of keys and values of one layer and which of them are free.  codes: 8-bit, with a step for each token and head."""

    def __init__(self, pages: int, page_size: int, heads: int, head_dim: int, dtype=torch.float16, codes: bool = False, device="cuda:0"):
        self.pages, self.page_size, self.heads, self.head_dim, self.dtype = pages, page_size, heads, head_dim, dtype
        self.kind = B.AWEQ_I8 if codes else DTYPES[dtype]
        new = lambda *shape, dtype: torch.empty(shape, dtype=dtype, device=device)
        self.k, self.v = (new(pages, heads, page_size, head_dim, dtype=torch.int8 if codes else dtype) for _ in range(2))
        self.k_step, self.v_step = (new(pages, heads, page_size, dtype=torch.float32) for _ in range(2)) if codes else (None, None)
        self.free = list(range(pages - 1, -1, -1))

    def take(self, tokens: int) -> List[int]:
        """Pages for that many tokens."""
        n = -(-tokens // self.page_size)
        if n > len(self.free):
            raise RuntimeError(f"{n} pages wanted, {len(self.free)} free")
        return [self.free.pop() for _ in range(n)]

    def give_back(self, pages: List[int]):
        self.free.extend(pages)

    def slots(self, pages: List[int], first: int, count: int) -> List[int]:
        """Where the tokens first .. first + count - 1 of a sequence with these pages go."""
        s = self.page_size
        return [pages[i // s] * s + i % s for i in range(first, first + count)]


def _check(name, t, dtype, shape, device, longer=False):
    """What the library reads by its address alone."""
    if t is None or t.device != device or t.dtype != dtype or t.dim() != len(shape) or not t.is_contiguous() or \
            (tuple(t.shape) < shape if longer else tuple(t.shape) != shape):
        raise ValueError(f"{name}: {dtype} {list(shape)}{' or longer' if longer else ''}, in one piece, on {device}")


class Sequences:
    """What a batch of sequences has in a cache, kept on the device: lengths, page tables and a stack of the cache's free pages, which a step takes from and
    gives back to without the host (all of them: the cache's own list is empty until give_back()).  Lengths and the stack's height are held twice, before and after a step: two steps, such as
    one that appends drafts and one that drops the rejected ones, end where they began, so that both can be captured in one graph."""

    def __init__(self, cache: PagedCache, batch: int, max_len: int, max_tokens: int, prefix_len: int = 0, max_drafts: int = 64):
        """max_len: tokens of a sequence; max_tokens: rows of a step; max_drafts: new tokens of a sequence in a step with masks."""
        self.cache, self.batch, self.prefix_len, self.max_tokens, self.max_drafts = cache, batch, prefix_len, max_tokens, max_drafts
        where = cache.k.device
        new = lambda *shape, dtype=torch.int32: torch.zeros(shape, dtype=dtype, device=where)
        self.table = new(batch, max(1, -(-max_len // cache.page_size)))
        free = cache.free
        self.free = new(cache.pages)
        self.free[:len(free)] = torch.tensor(free, dtype=torch.int32)
        self.counts = [torch.tensor([len(free)], dtype=torch.int32, device=where), new(1)]
        cache.free = []
        self.lengths, self.at = [new(batch), new(batch)], 0
        self.q_start, self.pos, self.slot = new(batch + 1), new(max_tokens), new(max_tokens, dtype=torch.int64)
        self.change = new(batch)
        self.mask = new(max_tokens, -(-max_drafts // 64), dtype=torch.int64)
        self.status = new(1)

    @property
    def lens(self):
        """Tokens of each sequence, after the last step."""
        return self.lengths[self.at]

    def step(self, change: torch.Tensor, tokens: int):
        """change [batch] int32: new tokens of each sequence, or (below 0) tokens that go; tokens: rows of the step, at least the new tokens.  Returns q_start, and pos and
        slot of the rows, buffers of this object's; nothing changes where the pages do not suffice (status ST_PAGES)."""
        c = self.cache
        _check("change", change, torch.int32, (self.batch,), c.k.device)
        if not 0 < tokens <= self.max_tokens:
            raise ValueError("one token at least, and no more than max_tokens")
        i, o = self.at, 1 - self.at
        pos, slot = self.pos[:tokens], self.slot[:tokens]
        B.aweq_step_plan(self.lengths[i], change, self.batch, c.page_size, c.pages, self.table, self.table.stride(0), self.table.shape[1], self.free, self.counts[i],
                         self.prefix_len, tokens, self.lengths[o], self.counts[o], self.q_start, pos, slot, self.status)
        self.at = o
        return self.q_start, pos, slot

    def draft(self, parent: torch.Tensor, max_q: int):
        """parent [tokens] int32: of each new token of the last step the place, among its sequence's, of the one that it goes on from, or -1.  Returns the masks
        [tokens, words], and writes the step's positions: a token's is its depth in the tree behind what its sequence has."""
        T = parent.shape[0]
        _check("parent", parent, torch.int32, (T,), self.cache.k.device)
        if not 0 < T <= self.max_tokens or not 0 < max_q <= self.max_drafts:
            raise ValueError("one token at least, and no more than max_tokens and max_drafts")
        B.aweq_tree_mask(parent, T, self.q_start, self.batch, max_q, self.lens, self.prefix_len, self.mask, self.mask.stride(0), self.pos, self.status)
        return self.mask[:T]

    def keep(self, kept: torch.Tensor, count: torch.Tensor, tokens: int) -> torch.Tensor:
        """kept [batch, most] int32: of each sequence the first count[b] are the places of the drafts that are accepted, in order.  Moves them to the front and returns the change
        that step() drops the others by."""
        c = self.cache
        if kept.dim() != 2 or kept.shape[1] < 1 or not 0 < tokens <= self.max_tokens:
            raise ValueError("kept: a row of places for each sequence; tokens: the step's rows")
        _check("kept", kept, torch.int32, (self.batch, kept.shape[1]), c.k.device)
        _check("count", count, torch.int32, (self.batch,), c.k.device)
        B.aweq_kv_keep(c.k, c.v, c.k_step, c.v_step, c.kind, c.pages, c.page_size, c.heads, c.head_dim, self.table, self.table.stride(0), self.lens, self.q_start,
                       self.batch, tokens, kept, kept.stride(0), count, self.change, self.status)
        return self.change

    def give_back(self):
        """The stack's pages to the cache's own list (waits for the device); the sequences take no more."""
        self.cache.free.extend(self.free[:int(self.counts[self.at].item())].tolist())
        self.counts[self.at].zero_()


class AttentionBlock:
    """qkv [(Hq + 2 Hk) D x hidden] and out [hidden x Hq D], each a QuantLinear or a Mx4Linear; buffers for max_tokens tokens of a step, allocated once."""

    def __init__(self, qkv, out, q_heads: int, cache: PagedCache, freq: Optional[torch.Tensor], rot: int, max_tokens: int,
                 interleaved: bool = False, gain: float = 1.0, q_norm=None, k_norm=None, eps: float = 1e-6, device="cuda:0"):
        D, Hk, where = cache.head_dim, cache.heads, cache.k.device
        if qkv.N != (q_heads + 2 * Hk) * D or out.K != q_heads * D:
            raise ValueError("the projections' sizes are not those of the heads")
        if D not in (64, 128, 256) or q_heads % Hk:
            raise ValueError("heads of 64, 128 or 256 values, and a whole number of query heads to a key head: the attention reads no others")
        if rot:
            _check("freq", freq, torch.float64, (rot // 2,), where)
        for name, w in (("q_norm", q_norm), ("k_norm", k_norm)):
            if w is not None:
                _check(name, w, torch.float32, (D,), where)
        self.qkv_layer, self.out_layer, self.q_heads, self.cache = qkv, out, q_heads, cache
        self.freq, self.rot, self.interleaved, self.gain, self.q_norm, self.k_norm, self.eps = freq, rot, interleaved, gain, q_norm, k_norm, eps
        self.max_tokens, self.device = max_tokens, device
        new = lambda *shape, dtype: torch.empty(shape, dtype=dtype, device=device)
        size = lambda layer: B.aweq_mx4_code_bytes(max_tokens, layer.K) if isinstance(layer, Mx4Linear) else B.aweq_panel_bytes(max_tokens, layer.K)
        self.xq = new(max(size(qkv), size(out)), dtype=torch.int8)
        self.x_scale = new(max([16] + [B.aweq_mx4_scale_bytes(max_tokens, layer.K) for layer in (qkv, out) if isinstance(layer, Mx4Linear)]), dtype=torch.uint8)
        self.step, self.zero, self.rowsum = new(max_tokens, dtype=torch.float32), new(max_tokens, dtype=torch.int32), new(max_tokens, dtype=torch.int32)
        self.qkv = new(max_tokens, qkv.N, dtype=cache.dtype)
        self.q = new(max_tokens, q_heads * D, dtype=cache.dtype)
        self.attended = new(max_tokens, q_heads * D, dtype=cache.dtype)
        self.y = new(max_tokens, out.N, dtype=cache.dtype)
        self.ws, self.kept = new(16, dtype=torch.uint8), []
        self.status = torch.zeros(1, dtype=torch.int32, device=device)

    def reserve(self, tokens, batch, max_q, prefix_len, max_len):
        """Scratch memory for steps of up to these bounds, so that none is allocated later."""
        self._scratch(B.aweq_prefix_attention_ws_most(tokens, self.q_heads, self.cache.heads, self.cache.head_dim, batch, max_q, prefix_len, max_len))

    def _scratch(self, need):
        """What was handed out before stays as it is: a captured graph writes there.  Twice as much each time, so that all of it is no more than the last."""
        if need > self.ws.numel():
            self.kept.append(self.ws)
            self.ws = torch.empty(max(need, 2 * self.ws.numel()), dtype=torch.uint8, device=self.device)

    def _product(self, layer, x, out):
        T, dt = x.shape[0], DTYPES[x.dtype]
        if isinstance(layer, Mx4Linear):
            B.aweq_mx4_gemm_tokens(x, dt, T, layer.K, x.stride(0), layer.factor, self.xq, self.x_scale, layer.codes, layer.scales, layer.N, layer.bias, out, dt,
                                   layer.N, self.status)
            return
        B.aweq_w8a8_gemm_tokens(x, dt, T, layer.K, x.stride(0), layer.inv_s, self.xq, self.step, self.zero, self.rowsum, layer.codes, layer.N,
                                layer.step_w, layer.zero_w, layer.w_group, layer.rowsum_w, layer.bias, out, dt, layer.N, self.status)

    def __call__(self, x, pos, slot, lens, table, q_start, max_len, max_q, prefix_table=None, prefix_len=0, mask=None):
        """x [T, hidden]: the step's tokens, sequence after sequence (q_start [B + 1], None: one each); pos [T] int32, slot [T] int64; lens [B]: the
        sequences' own keys with these tokens; table [B, ..]: their pages; mask [T, words] int64: which of its sequence's new tokens each one sees (None: those before
        it and itself).  Rows past q_start[B], of a step that is filled up, have no part in the others' results.  Returns [T, hidden], a buffer of the block's."""
        T, c = x.shape[0], self.cache
        if T > self.max_tokens or x.dtype != c.dtype:
            raise ValueError("more tokens than max_tokens, or another type than the cache's")
        batch, where = lens.shape[0], c.k.device
        if T == 0 or x.device != where or x.dim() != 2 or x.shape[1] != self.qkv_layer.K or x.stride(1) != 1:
            raise ValueError(f"x: [tokens, hidden], one token at least, each in one piece, on {where}")
        if self.rot:
            _check("pos", pos, torch.int32, (T,), where)
        _check("slot", slot, torch.int64, (T,), where)
        _check("lens", lens, torch.int32, (batch,), where)
        if q_start is not None:
            _check("q_start", q_start, torch.int32, (batch + 1,), where)
        if table.device != where or table.dtype != torch.int32 or table.dim() != 2 or table.shape[0] != batch or (table.shape[1] > 1 and table.stride(1) != 1):
            raise ValueError(f"table: int32 [sequences, pages], each row in one piece, on {where}")
        if prefix_len:
            _check("prefix_table", prefix_table, torch.int32, (-(-prefix_len // c.page_size),), where, longer=True)
        if mask is not None and (q_start is None or mask.device != where or mask.dtype != torch.int64 or mask.dim() != 2 or mask.shape[0] != T or
                                 64 * mask.shape[1] < min(max_q, T) or (mask.shape[1] > 1 and mask.stride(1) != 1)):
            raise ValueError(f"mask: int64 [{T}, a bit for each of max_q tokens], each row in one piece, on {where}, and q_start with it")
        max_len = min(max_len, table.shape[1] * c.page_size)   # (a view's pitch may be more than its pages)
        dt = DTYPES[x.dtype]
        Hq, Hk, D = self.q_heads, c.heads, c.head_dim
        width = self.qkv_layer.N
        self._product(self.qkv_layer, x, self.qkv)
        q, k, v = self.qkv[:T].split([Hq * D, Hk * D, Hk * D], 1)
        B.aweq_kv_append(q, k, v, dt, T, Hq, Hk, D, width, width, width, pos, self.freq, self.rot, self.interleaved, self.gain, self.q_norm, self.k_norm,
                         self.eps, self.q, Hq * D, c.k, c.v, c.k_step, c.v_step, c.kind, c.pages, c.page_size, slot, self.status)
        rows = T if q_start is None else min(T, batch * max_q)      # (the others of a step that is filled up are nobody's, and what was reserved is for no more)
        self._scratch(B.aweq_prefix_attention_ws(rows, Hq, Hk, D, batch, max_q, prefix_len, max_len))
        if q_start is not None:
            self.attended[:T].zero_()      # (rows behind the sequences' are nobody's, and are quantised like the others: not what an earlier step left there)
        if mask is None:
            B.aweq_prefix_attention(self.q, dt, rows, Hq, D, Hq * D, c.k, c.v, c.k_step, c.v_step, c.kind, c.pages, c.page_size, Hk, prefix_table, prefix_len,
                                    table, table.stride(0), lens, q_start, batch, max_len, max_q, D ** -0.5, self.attended, Hq * D, None, self.ws, self.status)
        else:
            B.aweq_tree_attention(self.q, dt, rows, Hq, D, Hq * D, c.k, c.v, c.k_step, c.v_step, c.kind, c.pages, c.page_size, Hk, prefix_table, prefix_len,
                                  table, table.stride(0), lens, q_start, batch, max_len, max_q, mask, mask.stride(0), D ** -0.5, self.attended, Hq * D, None,
                                  self.ws, self.status)
        self._product(self.out_layer, self.attended[:T], self.y)
        return self.y[:T]


def frequencies(rot: int, base: float = 10000.0, kind: int = B.ROPE_PLAIN, device="cuda:0", **scaling) -> Optional[torch.Tensor]:
    """The rotation's frequencies on the device; kind and scaling (factor, trained, low, high) as in aweq_rope_frequencies."""
    if rot == 0:
        return None
    host = torch.empty(rot // 2, dtype=torch.float64)
    B.aweq_rope_frequencies(rot, base, host, kind, **scaling)
    return host.to(device)


def calibrated(N, K, seed, tokens=512, dtype=torch.float16, device="cuda:0", mx4=False):
    """A random layer without a bias, calibrated on random activations with loud channels; mx4: its equalised weight in 4-bit floating point."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    x = torch.randn(tokens, K, generator=g, device=device)
    x[:, torch.randint(0, K, (max(1, K // 1000),), generator=g, device=device)] *= 50.0
    w = torch.randn(N, K, generator=g, device=device) * K ** -0.5
    buf = pipeline.LayerBuffers(tokens, K, N, torch.float16, want_out_i32=False, device=device)
    pipeline.calibrate_layer(x.half(), w.half(), None, buf, forward=False)
    return Mx4Linear.from_layer(buf) if mx4 else QuantLinear.from_layer(buf, correct=False)


def draft_steps(block, seqs, x, steps, tree, prefix_table, max_len):
    """Steps of a batch whose sequences each draft the tokens of `tree` (parents) and keep the path to the last of them; x [batch * tokens, hidden]."""
    m, dev = len(tree), x.device
    path, at = [], m - 1
    while at >= 0:
        path.append(at)
        at = tree[at]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)
    kept, count = ints([path[::-1]] * seqs.batch), ints([len(path)] * seqs.batch)
    more, parent = ints([m] * seqs.batch), ints(tree * seqs.batch)
    for _ in range(steps):
        q_start, pos, slot = seqs.step(more, x.shape[0])
        mask = seqs.draft(parent, m)
        y = block(x, pos, slot, seqs.lens, seqs.table, q_start, max_len, m, prefix_table, seqs.prefix_len, mask)
        seqs.step(seqs.keep(kept, count, x.shape[0]), x.shape[0])
        x = y.clone()
    return x, len(path)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--key-heads", type=int, default=32)
    ap.add_argument("--prefix", type=int, default=2048, help="tokens of the prompt that all sequences share")
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--codes", action="store_true", help="8-bit cache")
    ap.add_argument("--mx4", action="store_true", help="projections in 4-bit floating point")
    ap.add_argument("--draft", type=int, default=0, help="tokens of a tree that each sequence drafts in a step (0: one token a step)")
    a = ap.parse_args(argv)
    dev, D = "cuda:0", 128
    width = (a.heads + 2 * a.key_heads) * D
    most = a.steps * max(1, a.draft)        # tokens of a sequence, at most
    per = -(-most // 64) + 1
    cache = PagedCache(-(-a.prefix // 64) + a.batch * per, 64, a.key_heads, D, codes=a.codes, device=dev)
    block = AttentionBlock(calibrated(width, a.hidden, 1, mx4=a.mx4), calibrated(a.hidden, a.heads * D, 2, mx4=a.mx4), a.heads, cache, frequencies(D, device=dev), D,
                           max(a.prefix, a.batch * max(1, a.draft)), device=dev)
    ints = lambda v, dtype=torch.int32: torch.tensor(v, dtype=dtype, device=dev)
    # the prompt once, as one sequence of its own
    pages = cache.take(a.prefix)
    x = torch.randn(a.prefix, a.hidden, device=dev).half()
    if a.prefix:
        block(x, torch.arange(a.prefix, dtype=torch.int32, device=dev), ints(cache.slots(pages, 0, a.prefix), torch.int64), ints([a.prefix]), ints([pages]),
              ints([0, a.prefix]), a.prefix, a.prefix)
    if a.draft:
        # then the batch behind it, a tree each: pairs of tokens that go on from the same one
        seqs, shared = Sequences(cache, a.batch, most, a.batch * a.draft, a.prefix, a.draft), ints(pages)
        tree = [-1] + [(i - 1) // 2 for i in range(1, a.draft)]
        x = torch.randn(a.batch * a.draft, a.hidden, device=dev).half()
        block.reserve(a.batch * a.draft, a.batch, a.draft, a.prefix, most)
        torch.cuda.synchronize()
        began = time.perf_counter()
        x, path = draft_steps(block, seqs, x, a.steps, tree, shared, most)
        torch.cuda.synchronize()
        took = (time.perf_counter() - began) / a.steps
        print(f"{a.batch} sequences behind {a.prefix} shared tokens, {a.draft} drafted and {path} kept: {took * 1e6:.1f} us a step of the block, "
              f"status {int(block.status.item()) | int(seqs.status.item())}, output rms {x.float().pow(2).mean().sqrt().item():.3g}")
        return
    # then the batch behind it, a token each
    own = [cache.take(a.steps) for _ in range(a.batch)]
    table, shared = ints(own), ints(pages)
    plan = [(ints([a.prefix + i] * a.batch), ints([cache.slots(p, i, 1)[0] for p in own], torch.int64), ints([i + 1] * a.batch)) for i in range(a.steps)]
    x = torch.randn(a.batch, a.hidden, device=dev).half()
    block.reserve(a.batch, a.batch, 1, a.prefix, a.steps)
    torch.cuda.synchronize()
    began = time.perf_counter()
    for pos, slot, lens in plan:
        x = block(x, pos, slot, lens, table, None, a.steps, 1, shared, a.prefix).clone()
    torch.cuda.synchronize()
    took = (time.perf_counter() - began) / a.steps
    print(f"{a.batch} sequences behind {a.prefix} shared tokens: {took * 1e6:.1f} us a step of the block, status {int(block.status.item())}, "
          f"output rms {x.float().pow(2).mean().sqrt().item():.3g}")


if __name__ == "__main__":
    main()
