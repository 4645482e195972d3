"""diffqkv_extend on scores at the edges of their type: first tokens far below all others or at -inf, scores that are all far
from zero, and maxima that rise from tile to tile; against the definition in float64."""
import math

import pytest
import torch

from ragged import BF16, F32, HALF_STEP, Step

pytestmark = pytest.mark.gpu

TILE = 128  # tokens


@pytest.fixture(scope="module")
def api():
    from paper_2501_13629_b200 import api as _api
    return _api


def check(step, out, lse, scale):
    """Bounds as in ragged.check_extend, with the size of the scores taken per row over the tokens whose weight is at least
    1e-30: the others' weights are zero or add less than t 1e-30 to the result, whatever their scores are off by (scores
    below -10^4 are off by less than a thousandth of themselves)."""
    assert bool(torch.isfinite(out).all()) and not bool(torch.isnan(lse).any())
    for b, (past, n) in enumerate(zip(step.past, step.new)):
        lo, t = step.cu_host[b], step.total[b]
        q = step.q[lo:lo + n].double()
        k = step.k_tok[b].double().repeat_interleave(step.n_q // step.n_k, 1)
        v = step.v_tok[b].double().repeat_interleave(step.n_q // step.n_v, 1)
        x = torch.einsum("ihd,jhd->ihj", q, k) * scale
        hidden = torch.arange(t, device="cuda")[None] > past + torch.arange(n, device="cuda")[:, None]
        x = torch.where(x * math.log2(math.e) < -torch.finfo(F32).max, -math.inf, x)  # beyond fp32 in units of log 2
        x = x.masked_fill(hidden[:, None], -math.inf)
        ref_lse = torch.logsumexp(x, 2)
        none = ref_lse == -math.inf  # such a row has nothing
        assert bool((out[lo:lo + n][none] == 0).all()) and bool((lse[lo:lo + n][none] == -math.inf).all())
        ref_lse = ref_lse.masked_fill(none, 0.0)
        p = torch.exp(x - ref_lse[..., None])
        size = torch.einsum("ihd,jhd->ihj", q.abs(), k.abs()) * scale
        big = torch.where(p >= 1e-30, size, 0.0).amax(2).clamp(min=1.0)
        ref, mean_abs = torch.einsum("ihj,jhd->ihd", p, v), torch.einsum("ihj,jhd->ihd", p, v.abs())
        score = (step.d_qk + 16) * 2.0 ** -24 * big
        weight = (2 * score + (t + 16) * 2.0 ** -24 + (HALF_STEP[BF16] if step.dtype == BF16 else 0.0))[..., None]
        bound = weight * mean_abs * (1 + weight) + 1e-25
        bound = bound + HALF_STEP[out.dtype] * (ref.abs() + bound)
        err = (out[lo:lo + n].double() - ref).abs()
        assert bool((err <= bound).all()), f"sequence {b}: {float((err / bound).max()):.2f} times the bound"
        bound = score + (t + 16) * 2.0 ** -24 + 2.0 ** -22 * ref_lse.abs()
        err = (lse[lo:lo + n].double().masked_fill(none, 0.0) - ref_lse).abs()
        assert bool((err <= bound).all()), f"sequence {b}: lse {float((err / bound).max()):.2f} times the bound"


def run(api, step, scale=1.0):
    out = torch.empty((step.total_q, step.n_q, step.d_v), dtype=F32, device="cuda")
    lse = torch.empty((step.total_q, step.n_q), dtype=F32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.diffqkv_extend(step.q, step.cu, step.cache, step.n_k, step.n_v, scale, out=out, lse=lse, dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    check(step, out, lse, scale)


def made(api, past, new, heads, dims, dtype, level, seed):
    """Scores of about one in size around level(token numbers): the first channel of every query is 1."""
    step = Step(api, past, new, *heads, *dims, dtype=dtype, seed=seed)
    spread = dims[0] ** -0.25
    step.q = (step.q.float() * spread).to(dtype)
    step.q[..., 0] = 1.0
    for b, t in enumerate(step.total):
        step.k_tok[b] = (step.k_tok[b].float() * spread).to(dtype)
        step.k_tok[b][:, :, 0] = level(torch.arange(t, device="cuda")).to(dtype)[:, None]
    return step.fill()


STEPS = {"one token": ([5], [1]), "a few": ([126, 700], [3, 1]), "long caches": ([3000, 20, 9000], [2, 5, 1]),
         "long chunks": ([0, 300], [140, 70])}


@pytest.mark.parametrize("low", [-math.inf, -3.38e38, -1e7, -1e5, -3e4, -1e3])
@pytest.mark.parametrize("others", [0.0, -300.0])
@pytest.mark.parametrize("step", STEPS)
@pytest.mark.parametrize("dims,dtype", [((128, 128), BF16), ((64, 64), BF16), ((64, 128), BF16), ((64, 64), F32), ((96, 64), F32)])
def test_first_tokens_far_below(api, low, others, step, dims, dtype):
    """The first token of every tile has a score of -inf or far below all others' (and no weight worth a number)."""
    level = lambda j: torch.where(j % TILE == 0, low, others)  # noqa: E731
    run(api, made(api, *STEPS[step], (16, 2, 4), dims, dtype, level, 1))


@pytest.mark.parametrize("rise", [20.0, 60.0, 2000.0, -60.0])
@pytest.mark.parametrize("step", STEPS)
@pytest.mark.parametrize("dims,dtype", [((128, 128), BF16), ((64, 64), BF16), ((64, 64), F32)])
def test_maxima_move_from_tile_to_tile(api, rise, step, dims, dtype):
    level = lambda j: -800.0 + rise * (j // TILE)  # noqa: E731
    run(api, made(api, *STEPS[step], (32, 4, 8), dims, dtype, level, 2))


@pytest.mark.parametrize("level", [-1e4, 1e4])
@pytest.mark.parametrize("step", STEPS)
def test_scores_far_from_zero(api, level, step):
    run(api, made(api, *STEPS[step], (8, 4, 2), (128, 128), BF16, lambda j: torch.full_like(j, level, dtype=F32), 3))


@pytest.mark.parametrize("dims,dtype", [((128, 128), BF16), ((64, 64), BF16), ((64, 64), F32), ((96, 64), F32), ((96, 64), BF16)])
@pytest.mark.parametrize("bad", [-math.inf, math.nan, math.inf])
def test_keys_that_are_not_finite(api, dims, dtype, bad):
    """All visible keys at -inf: nothing; at NaN or +inf: NaN; rows that see numbers beside -inf: the numbers."""
    for new in ([1, 2], [4, 150]):
        step = made(api, [140, 0], new, (8, 2, 4), dims, dtype, lambda j: torch.where(j < 142, bad, 1.0), 4)
        out = torch.empty((step.total_q, 8, step.d_v), dtype=F32, device="cuda")
        lse = torch.empty((step.total_q, 8), dtype=F32, device="cuda")
        api.diffqkv_extend(step.q, step.cu, step.cache, 2, 4, 1.0, out=out, lse=lse)
        torch.cuda.synchronize()
        if bad == -math.inf:
            check(step, out, lse, 1.0)
        else:
            assert bool(out.isnan().all()) and bool(lse.isnan().all())


@pytest.mark.parametrize("seed", range(10))
@pytest.mark.parametrize("spread", [10.0, 300.0])
def test_heavy_tails(api, seed, spread):
    """Tokens' levels drawn from a Cauchy distribution: maxima jump anywhere, by anything, up and not at all."""
    g = torch.Generator("cuda").manual_seed(seed)

    def level(j):
        u = torch.rand(j.shape, generator=g, device="cuda", dtype=torch.float64)
        return (spread * torch.tan(math.pi * (u - 0.5))).clamp(-1e6, 1e4)

    heads = [(32, 4, 8), (16, 8, 2), (12, 2, 6), (16, 1, 1), (32, 4, 16)][seed % 5]
    dims = [(128, 128), (64, 64), (64, 128)][seed % 3]
    run(api, made(api, [2000, 40, 300, 5000, 0, 129], [1, 3, 2, 1, 4, 150 if seed % 2 else 2], heads, dims, BF16, level, seed))
