"""Ragged steps over a cache for the tests: seeded inputs, the definitions in float64, and bounds from the arithmetic."""
import math

import torch

BF16, F32 = torch.bfloat16, torch.float32
HALF_STEP = {BF16: 2.0 ** -8, F32: 2.0 ** -24}  # rounding to the type, relative


def ints(x, device="cuda"):
    return torch.tensor(x, dtype=torch.int32, device=device)


class Step:
    """Pools, table and lengths of a ragged step.  layout: "paged" (head-major pages), "token" (token-major pages),
    "flat" (contiguous per sequence).  Everything no sequence owns, the slots behind its last token included, is NaN."""

    def __init__(self, api, past, new, n_q, n_k, n_v, d_qk, d_v, dtype=BF16, page=16, layout="paged", pad=0, seed=0,
                 room=0, k_std=1.0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.past, self.new, self.page, self.layout, self.dtype = list(past), list(new), page, layout, dtype
        self.n_q, self.n_k, self.n_v, self.d_qk, self.d_v = n_q, n_k, n_v, d_qk, d_v
        B = len(self.past)
        self.total = [p + n for p, n in zip(self.past, self.new)]
        cu = [0]
        for n in self.new:
            cu.append(cu[-1] + n)
        self.rows, self.total_q, self.cu_host = cu[-1], cu[-1] + pad, cu
        self.cu = ints(cu)
        rand = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=F32).to(dtype)  # noqa: E731
        self.q = rand(self.total_q, n_q, d_qk)
        self.q[self.rows:] = math.nan
        self.k_tok = [(rand(t, n_k, d_qk).float() * k_std).to(dtype) for t in self.total]  # tokens of every sequence
        self.v_tok = [rand(t, n_v, d_v) for t in self.total]
        longest = max(self.total) + room
        if layout == "flat":
            S = longest
            self.k = torch.full((B, n_k, S, d_qk), math.nan, dtype=dtype, device="cuda")
            self.v = torch.full((B, n_v, S, d_v), math.nan, dtype=dtype, device="cuda")
            self.table, self.max_seqlen = None, S
        else:
            per = [-(-t // page) for t in self.total]
            row = max(1, -(-longest // page))
            pages = sum(per) + 2
            order = torch.randperm(pages, generator=g, device="cuda").cpu()
            self.table = torch.full((B, row), -1, dtype=torch.int32)
            at = 0
            for b, n in enumerate(per):
                self.table[b, :n] = order[at:at + n].int()
                at += n
            self.table = self.table.cuda()
            shape = (lambda h, d: (pages, h, page, d)) if layout == "paged" else (lambda h, d: (pages, page, h, d))
            self.k = torch.full(shape(n_k, d_qk), math.nan, dtype=dtype, device="cuda")
            self.v = torch.full(shape(n_v, d_v), math.nan, dtype=dtype, device="cuda")
            self.max_seqlen = row * page
        if layout == "token":
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)  # [page, head, slot, d] with token strides
        self.lens = ints(self.past)
        self.cache = api.KVCache(self.k, self.v, self.lens, self.max_seqlen, page_table=self.table,
                                 page_size=0 if self.table is None else page)

    def place(self, b, start, stop):
        """(block, slot) indexes of tokens start .. stop - 1 of sequence b."""
        t = torch.arange(start, stop, device="cuda")
        if self.layout == "flat":
            return torch.full_like(t, b), t
        return self.table[b].long()[t // self.page], t % self.page

    def fill(self, whole=True):
        """Write the tokens into the pools: all of them, or only those cached before the step."""
        for b in range(len(self.past)):
            n = self.total[b] if whole else self.past[b]
            blk, slot = self.place(b, 0, n)
            self.k[blk, :, slot] = self.k_tok[b][:n]
            self.v[blk, :, slot] = self.v_tok[b][:n]
        return self


def attend64(q, k, v, scale, first):
    """Row i of q [n, n_q, d] sees tokens 0 .. first + i of k [t, n_k, d], v [t, n_v, d]: (out, lse, sum p |v| / sum p,
    largest sum |q k| scale), float64."""
    n, n_q = q.shape[0], q.shape[1]
    k = k.double().repeat_interleave(n_q // k.shape[1], 1)
    v = v.double().repeat_interleave(n_q // v.shape[1], 1)
    x = torch.einsum("ihd,jhd->hij", q.double(), k) * scale
    big = torch.einsum("ihd,jhd->hij", q.double().abs(), k.abs()).amax() * abs(scale)
    hidden = torch.arange(k.shape[0], device=q.device)[None] > first + torch.arange(n, device=q.device)[:, None]
    x = x.masked_fill(hidden, -math.inf)
    lse = torch.logsumexp(x, 2)
    p = torch.exp(x - lse[..., None])
    return (torch.einsum("hij,jhd->ihd", p, v), lse.T, torch.einsum("hij,jhd->ihd", p, v.abs()), float(big))


def check_extend(step, out, lse, scale):
    """Bounds, all from the arithmetic.  Scores: d products summed in fp32 from exact products, error <= d 2^-24 sum|q k|
    scale, plus a few roundings (scale, maximum, exponent: 16 steps).  A weight's relative error is the score's error
    twice over (its own and the maximum's), plus half a step of bf16 where the weights are rounded for the second
    product; that product and the sum of weights add t roundings of fp32.  The result is rounded once."""
    for b, (past, n) in enumerate(zip(step.past, step.new)):
        lo = step.cu_host[b]
        if n == 0:
            continue
        ref, ref_lse, mean_abs, big = attend64(step.q[lo:lo + n], step.k_tok[b], step.v_tok[b], scale, past)
        t = step.total[b]
        score = (step.d_qk + 16) * 2.0 ** -24 * max(big, 1.0)
        weight = 2 * score + (t + 16) * 2.0 ** -24 + (HALF_STEP[BF16] if step.dtype == BF16 else 0.0)
        bound = weight * mean_abs * (1 + weight)
        bound = bound + HALF_STEP[out.dtype] * (ref.abs() + bound)
        err = (out[lo:lo + n].double() - ref).abs()
        assert torch.isfinite(out[lo:lo + n]).all(), f"sequence {b}"
        assert bool((err <= bound).all()), f"sequence {b}: {float((err / bound).max()):.2f} times the bound"
        if lse is not None:
            bound_lse = score + (t + 16) * 2.0 ** -24 + 2.0 ** -22 * ref_lse.abs()
            err = (lse[lo:lo + n].double() - ref_lse).abs()
            assert bool((err <= bound_lse).all()), f"sequence {b}: lse {float((err / bound_lse).max()):.2f} times the bound"
