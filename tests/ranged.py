"""Steps whose rows do not see all tokens before them, for the tests: the definitions in float64, and bounds from the
arithmetic."""
import math

import torch

from ragged import BF16, F32, HALF_STEP, Step, ints  # noqa: F401


def visible(past, n, t, window=None, sinks=0):
    """[n, t]: row i at position past + i sees token j."""
    i = past + torch.arange(n, device="cuda")[:, None]
    j = torch.arange(t, device="cuda")[None]
    sees = j <= i
    return sees if window is None else sees & ((j < sinks) | (j > i - window))


def attend64(q, k, v, scale, sees):
    """(out, lse, sum p |v|, largest sum |q k| scale over what is seen), float64; q [n, n_q, d], sees [n, t]."""
    n_q = q.shape[1]
    k = k.double().repeat_interleave(n_q // k.shape[1], 1)
    v = v.double().repeat_interleave(n_q // v.shape[1], 1)
    some = sees.any(0)  # tokens that nobody sees may hold anything
    k, v, sees = k[some], v[some], sees[:, some]
    x = torch.einsum("ihd,jhd->hij", q.double(), k) * scale
    big = (torch.einsum("ihd,jhd->hij", q.double().abs(), k.abs()) * abs(scale)).masked_fill(~sees, 0.0).amax()
    x = x.masked_fill(~sees, -math.inf)
    lse = torch.logsumexp(x, 2)
    p = torch.exp(x - lse[..., None])
    return torch.einsum("hij,jhd->ihd", p, v), lse.T, torch.einsum("hij,jhd->ihd", p, v.abs()), float(big)


def check(step, out, lse, scale, window=None, sinks=0, joined=False, only=None):
    """Bounds as in ragged.check_extend: a score of d exact products summed in fp32 is off by d 2^-24 sum |q k| scale and a
    few roundings (16 steps); a weight by twice that and, where weights are rounded for the second product, half a step of
    bf16; sums over t tokens add t roundings.  A row joined from two parts by their log-sum-exps in units of log 2 (joined):
    each of these is rounded once (half a step of 2^-23 of its size) and goes through an exponential good to 2^-22, and so
    does their difference: 2^-21 + |lse| 2^-22 in a part's weight."""
    for b, (past, n) in enumerate(zip(step.past, step.new)):
        lo, t = step.cu_host[b], step.total[b]
        if n == 0 or (only is not None and b not in only):
            continue
        ref, ref_lse, mean_abs, big = attend64(step.q[lo:lo + n], step.k_tok[b], step.v_tok[b], scale,
                                               visible(past, n, t, window, sinks))
        score = (step.d_qk + 16) * 2.0 ** -24 * max(big, 1.0)
        weight = 2 * score + (t + 16) * 2.0 ** -24 + (HALF_STEP[BF16] if step.dtype == BF16 else 0.0)
        if joined:
            weight = (weight + 2.0 ** -21 + 2.0 ** -22 * ref_lse.abs() * 1.4427)[..., None]
        bound = weight * mean_abs * (1 + weight)
        bound = bound + HALF_STEP[out.dtype] * (ref.abs() + bound)
        got = out[lo:lo + n].double()
        assert bool(torch.isfinite(got).all()), f"sequence {b}"
        err = (got - ref).abs()
        assert bool((err <= bound).all()), f"sequence {b}: {float((err / bound).max()):.2f} times the bound"
        if lse is not None:
            bound = score + (t + 16) * 2.0 ** -24 + 2.0 ** -21 * ref_lse.abs() + (2.0 ** -21 if joined else 0.0)
            err = (lse[lo:lo + n].double() - ref_lse).abs()
            assert bool((err <= bound).all()), f"sequence {b}: lse {float((err / bound).max()):.2f} times the bound"


def forget(step, window, sinks):
    """Tokens that no row of the step sees become NaN, and pages that hold none but such are taken away (entry -1)."""
    for b, (past, n) in enumerate(zip(step.past, step.new)):
        low = max(0, past + 1 - window) if n else step.total[b]
        first = sinks if n else 0
        if low <= first:
            continue
        blk, slot = step.place(b, first, low)
        step.k[blk, :, slot] = math.nan
        step.v[blk, :, slot] = math.nan
        if step.table is not None:
            gone = slice(-(-first // step.page), low // step.page if n else None)
            step.table[b, gone] = -1
    return step
