"""diffqkv_extend_window: ragged chunks within a sliding window and to the first tokens, against the definition in float64."""
import math
import random

import pytest
import torch

from ragged import BF16, F32, Step, ints
from ranged import HALF_STEP, attend64, check, forget

pytestmark = pytest.mark.gpu

HEADS = {"32/4/8": (32, 4, 8), "16/2/4": (16, 2, 4), "8/8/8": (8, 8, 8), "8/4/2": (8, 4, 2), "12/2/4": (12, 2, 4),
         "6/2/3": (6, 2, 3), "16/1/1": (16, 1, 1), "32/4/16": (32, 4, 16), "20/4/4": (20, 4, 4)}


@pytest.fixture(scope="module")
def api():
    from paper_2501_13629_b200 import api as _api
    return _api


def run(api, step, window, sinks, scale=None, out_dtype=None, want_lse=True, workspace=None, stream=None):
    scale = step.d_qk ** -0.5 if scale is None else scale
    out = torch.full((step.total_q, step.n_q, step.d_v), 77.0, dtype=out_dtype or step.dtype, device="cuda")
    lse = torch.full((step.total_q, step.n_q), 77.0, dtype=F32, device="cuda") if want_lse else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.diffqkv_extend_window(step.q, step.cu, step.cache, step.n_k, step.n_v, scale, window, sinks=sinks, out=out, lse=lse,
                              dev_status=status, workspace=workspace, stream=stream)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    assert bool((out[step.rows:] == 77.0).all())  # rows behind the last chunk stay as they were
    if want_lse:
        assert bool((lse[step.rows:] == 77.0).all())
    check(step, out, lse, scale, window, sinks)
    return out, lse


PAST = [0, 5, 130, 127, 700, 0, 64, 1023, 300, 0]
NEW = [1, 1, 4, 1, 33, 129, 0, 65, 257, 300]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dims", [(128, 128), (64, 64), (64, 128)])
@pytest.mark.parametrize("window,sinks", [(100, 4), (200, 0)])
def test_ragged_chunks_in_pages(api, heads, dims, window, sinks):
    """Chunks of every kind in one batch; pages and tokens that no row sees are not there."""
    step = Step(api, PAST, NEW, *HEADS[heads], *dims, page=16, pad=3, seed=len(heads)).fill()
    run(api, forget(step, window, sinks), window, sinks)


@pytest.mark.parametrize("window", [1, 2, 17, 127, 128, 129, 256, 300, 1000, 5000])
@pytest.mark.parametrize("sinks", [0, 1, 4, 127, 128, 129, 200, 1500])
def test_windows_and_first_tokens(api, window, sinks):
    step = Step(api, PAST, NEW, 8, 2, 4, 64, 64, page=16, pad=1, seed=window + sinks).fill()
    run(api, forget(step, window, sinks), window, sinks)


@pytest.mark.parametrize("page,layout", [(8, "paged"), (16, "token"), (32, "paged"), (64, "paged"), (128, "paged"),
                                         (256, "paged"), (16, "flat"), (24, "paged"), (4, "paged")])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_page_sizes_and_layouts(api, page, layout, dtype):
    """Pages that end inside a tile, tiles inside a page, token-major pools, no pages, and sizes only the plain kernel takes."""
    step = Step(api, [300, 0, 129, 17, 900], [70, 140, 2, 1, 3], 8, 2, 4, 128, 128, dtype=dtype, page=page, layout=layout,
                seed=page, room=40)
    run(api, forget(step.fill(), 90, 10), 90, 10)


@pytest.mark.parametrize("dtype,out_dtype", [(BF16, F32), (BF16, BF16), (F32, F32), (F32, BF16)])
def test_types(api, dtype, out_dtype):
    step = Step(api, [50, 400, 600], [200, 3, 0], 16, 2, 4, 64, 64, dtype=dtype, seed=3).fill()
    run(api, forget(step, 70, 3), 70, 3, out_dtype=out_dtype, want_lse=out_dtype == F32)


@pytest.mark.parametrize("dims", [(32, 32), (96, 80), (128, 256), (256, 128), (8, 512), (192, 128), (128, 64)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_other_head_dimensions(api, dims, dtype):
    step = Step(api, [33, 0, 500], [5, 40, 1], 4, 2, 4, *dims, dtype=dtype, seed=dims[0]).fill()
    run(api, forget(step, 20, 2), 20, 2)


@pytest.mark.parametrize("choice", [1, 2])
@pytest.mark.parametrize("heads", ["32/4/8", "6/2/3", "16/1/1"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window,sinks", [(1, 0), (150, 0), (150, 7), (700, 300)])
def test_kernels_on_fmas(api, choice, heads, dtype, window, sinks):
    """The kernels that take what the tensor cores do not: many rows, and few over a long cache."""
    api.extend_kernel(choice)
    try:
        step = Step(api, [0, 5, 130, 700, 0], [1, 4, 33, 129, 0], *HEADS[heads], 64, 128, dtype=dtype, seed=21).fill()
        run(api, forget(step, window, sinks), window, sinks)
        assert api.last_extend_kernel() == choice
        step = Step(api, [3000, 90, 1024], [2, 1, 1], *HEADS[heads], 128, 64, dtype=dtype, seed=22, pad=2).fill()
        run(api, forget(step, window, sinks), window, sinks)
    finally:
        api.extend_kernel(0)


@pytest.mark.parametrize("past", [0, 1, 4000, 4095, 4096, 20000, 20001])
@pytest.mark.parametrize("window,sinks", [(4096, 4), (1000, 0), (130, 64)])
def test_single_tokens_over_long_caches(api, past, window, sinks):
    step = Step(api, [past, 77, past // 2], [1, 1, 5], 32, 4, 8, 128, 128, seed=past).fill()
    run(api, forget(step, window, sinks), window, sinks)


@pytest.mark.parametrize("heads", ["32/4/8", "6/2/3", "8/8/8"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (31, 1), (500, 130), (1500, 0)])
def test_long_chunks(api, heads, window, sinks):
    """Many row tiles whose windows begin in different tiles, cut wherever a block's share ends."""
    step = Step(api, [100, 0, 2500, 60], [1100, 1, 700, 9], *HEADS[heads], 64, 64, page=64, seed=6, pad=1).fill()
    run(api, forget(step, window, sinks), window, sinks)


@pytest.mark.parametrize("heads", ["32/4/8", "6/2/3", "8/8/8", "16/1/1", "12/2/4"])
@pytest.mark.parametrize("window,sinks", [(7, 0), (100, 70), (400, 1)])
@pytest.mark.parametrize("new", [[15, 16, 17], [31, 1, 33], [21, 22, 43, 2], [63, 64, 65], [127, 128, 129, 5], [160], [0, 255, 1]])
def test_chunks_around_what_is_few(api, heads, window, sinks, new):
    """Rows that fill the blocks of the kernel of few rows, one less and one more."""
    step = Step(api, [50 + 90 * i for i in range(len(new))], new, *HEADS[heads], 64, 128, page=32, seed=sum(new), pad=2).fill()
    run(api, forget(step, window, sinks), window, sinks)


@pytest.mark.parametrize("past,new", [(PAST, NEW), ([0, 900], [600, 700]), ([3, 17], [2, 1]), ([3000] * 4, [1] * 4)])
def test_a_window_over_the_whole_cache(api, past, new):
    """What extend gives: long chunks by its kernels, few rows by others."""
    step = Step(api, past, new, 16, 2, 4, 128, 128, seed=8, pad=2).fill()
    out = torch.empty((step.total_q, 16, 128), dtype=BF16, device="cuda")
    api.diffqkv_extend(step.q, step.cu, step.cache, 2, 4, 0.1, out=out)
    check(step, out, None, 0.1)
    for window, sinks in ((step.max_seqlen, 0), (step.max_seqlen - 2, 2), (2 ** 31 - 1, 2 ** 31 - 1), (1, 2 ** 31 - 1), (2 ** 31 - 1, 1)):
        got, _ = run(api, step, window, sinks, scale=0.1)
        if len(past) == 2 and new[0] > 500:
            assert torch.equal(got[:step.rows], out[:step.rows])


@pytest.mark.parametrize("window", [1300, 1023, 1024])
def test_a_wide_window_agrees_with_extend(api, window):
    """A window that hides nothing of what is cached, but less than the cache could hold."""
    step = Step(api, PAST, NEW, 16, 2, 4, 128, 128, seed=8, pad=2, room=500).fill()
    run(api, step, window, 0)


@pytest.mark.parametrize("k_std", [10.0, 40.0])
@pytest.mark.parametrize("new", [[3, 1], [140, 300]])
def test_peaked_scores(api, new, k_std):
    """References are raised often, most weights vanish."""
    step = Step(api, [900, 240], new, 8, 2, 4, 128, 128, seed=4, k_std=k_std).fill()
    run(api, forget(step, 300, 5), 300, 5)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [1, 4, 90])
def test_rows_that_see_nothing_but_minus_infinity(api, dtype, new):
    """All scores within the window are -inf; the finite ones lie in front of it."""
    step = Step(api, [600], [new], 4, 2, 2, 64, 64, dtype=dtype, seed=2)
    step.q[:] = step.q.abs() + 0.1
    step.k_tok[0][300:] = -math.inf
    step.fill()
    out, lse = torch.empty((new, 4, 64), dtype=F32, device="cuda"), torch.empty((new, 4), dtype=F32, device="cuda")
    api.diffqkv_extend_window(step.q, step.cu, step.cache, 2, 2, 0.125, 200, out=out, lse=lse)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    api.diffqkv_extend_window(step.q, step.cu, step.cache, 2, 2, 0.125, 200, sinks=4, out=out, lse=lse)
    x = torch.einsum("ihd,jhd->ihj", step.q.double(), step.k_tok[0][:4].double().repeat_interleave(2, 1)) * 0.125
    assert bool(((lse.double() - x.logsumexp(2)).abs() <= 80 * 2.0 ** -24 * 64).all())


def test_nan_in_what_a_row_sees_stays_with_it(api):
    step = Step(api, [500, 500], [2, 2], 4, 2, 2, 128, 128, seed=2)
    step.k_tok[1][450] = math.nan
    step.fill()
    out = torch.empty((4, 4, 128), dtype=BF16, device="cuda")
    api.diffqkv_extend_window(step.q, step.cu, step.cache, 2, 2, 0.1, 100, out=out)
    assert bool(torch.isfinite(out[:2]).all()) and bool(torch.isnan(out[2:]).all())


def test_repeats_bit_for_bit_and_with_any_workspace(api):
    step = forget(Step(api, [3000, 10, 700], [2, 1, 600], 32, 4, 8, 128, 128, seed=5).fill(), 900, 4)
    first, lse = run(api, step, 900, 4)
    nbytes = api.diffqkv_extend_window_workspace_bytes(api.make_shape(3, 32, 4, 8, 128, 128, BF16, BF16, 1.0), step.total_q)
    for fill in (0, 255):
        ws = torch.full((nbytes,), fill, dtype=torch.uint8, device="cuda")
        again, lse2 = run(api, step, 900, 4, workspace=ws)
        assert torch.equal(first, again) and torch.equal(lse, lse2)


def test_sequences_that_do_not_fit(api):
    """Reported and skipped; the others are as they would be."""
    for dtype, dims in ((BF16, (128, 128)), (F32, (64, 64)), (BF16, (96, 80))):
        step = Step(api, [300, 200, 400], [3, 40, 1], 8, 2, 4, *dims, dtype=dtype, seed=7, pad=1).fill()
        step.lens[1] = -1
        out = torch.full((step.total_q, 8, dims[1]), 77.0, dtype=dtype, device="cuda")
        status = ints([0])
        api.diffqkv_extend_window(step.q, step.cu, step.cache, 2, 4, 0.1, 128, sinks=2, out=out, dev_status=status)
        assert int(status.item()) == 1 << api.ERR_INDEX
        assert bool((out[3:43] == 77.0).all()) and bool((out[44:] == 77.0).all())
        check(step, out, None, 0.1, 128, 2, only=(0, 2))


@pytest.mark.parametrize("new,bad,rows", [([1, 2, 1], 1, slice(1, 3)), ([1, 0, 1], 1, slice(0, 0)), ([2, 1, 1], 0, slice(0, 2))])
def test_a_few_rows_in_all_that_do_not_fit(api, new, bad, rows):
    """Steps that one kernel takes alone."""
    step = Step(api, [300, 200, 400], new, 8, 2, 4, 128, 128, seed=7, pad=1).fill()
    step.lens[bad] = step.max_seqlen + 1
    out, status = torch.full((step.total_q, 8, 128), 77.0, dtype=BF16, device="cuda"), ints([0])
    api.diffqkv_extend_window(step.q, step.cu, step.cache, 2, 4, 0.1, 128, sinks=2, out=out, dev_status=status)
    assert int(status.item()) == 1 << api.ERR_INDEX
    assert bool((out[rows] == 77.0).all()) and bool((out[step.rows:] == 77.0).all())
    check(step, out, None, 0.1, 128, 2, only=[b for b in range(3) if b != bad])


@pytest.mark.parametrize("batch", [300, 700, 1200])
def test_more_sequences_than_threads(api, batch):
    r = random.Random(batch)
    past = [r.choice([0, r.randint(0, 300)]) for _ in range(batch)]
    new = [r.choice([0, 1, 1, 2, 40]) if b % 9 else 1 for b in range(batch)]
    step = Step(api, past, new, 8, 2, 4, 64, 64, seed=batch, pad=2).fill()
    run(api, forget(step, 60, 3), 60, 3)


def test_offsets_past_32_bits(api):
    """A pool of more than 2^32 bytes and elements, of which a window lies at the end."""
    past, n_k, d = 2_100_000, 16, 128
    k, v = (torch.empty((1, n_k, past + 128, d), dtype=BF16, device="cuda") for _ in range(2))  # 4.3 G elements each
    window, rows = 200, 3
    for x in (k, v):
        x[:, :, :4].normal_()
        x[:, :, past - window:past + rows].normal_()
    q = torch.randn((rows, n_k, d), device="cuda").to(BF16)
    cache = api.KVCache(k, v, ints([past]), past + rows)
    out = torch.empty_like(q)
    api.diffqkv_extend_window(q, ints([0, rows]), cache, n_k, n_k, 0.1, window, sinks=4, out=out)
    seen = torch.cat([torch.arange(4, device="cuda"), torch.arange(past - window + 1, past + rows, device="cuda")])
    pos = past + torch.arange(rows, device="cuda")[:, None]
    sees = (seen[None] <= pos) & ((seen[None] < 4) | (seen[None] > pos - window))
    kd, vd = (x[0][:, seen].double().transpose(0, 1) for x in (k, v))
    ref, _, mean_abs, big = attend64(q, kd, vd, 0.1, sees)
    weight = 2 * (d + 16) * 2.0 ** -24 * max(big, 1.0) + (len(seen) + 16) * 2.0 ** -24 + HALF_STEP[BF16]
    bound = weight * mean_abs * (1 + weight)
    bound = bound + HALF_STEP[BF16] * (ref.abs() + bound)
    assert bool(((out.double() - ref).abs() <= bound).all())


def test_rows_given_to_many_sequences_at_once(api):
    """cu_q goes back and forth, so that every other sequence has all rows: far more work than the step's rows can be.  It is
    reported, and left out."""
    n, pairs, tokens = 32768, 300, 1 << 20
    q = torch.zeros((n, 8, 64), dtype=BF16, device="cuda")
    pool = torch.zeros((2, 8, 16, 64), dtype=BF16, device="cuda")
    table = torch.zeros((2 * pairs, tokens // 16), dtype=torch.int32, device="cuda")
    cache = api.KVCache(pool, pool.clone(), ints([tokens - n] * (2 * pairs)), tokens, page_table=table, page_size=16)
    status, out = ints([0]), torch.full((n, 8, 64), 77.0, dtype=BF16, device="cuda")
    api.diffqkv_extend_window(q, ints([0, n] * pairs + [0]), cache, 8, 8, 0.1, tokens - 1, out=out, dev_status=status)
    assert int(status.item()) == 1 << api.ERR_INDEX and api.last_extend_kernel() == 3
    assert bool((out == 77.0).all())


def test_a_missing_page_inside_the_window_is_reported(api):
    step = Step(api, [300], [3], 8, 2, 4, 128, 128, seed=7).fill()
    out, status = torch.empty((3, 8, 128), dtype=BF16, device="cuda"), ints([0])
    step.table[0, 5] = -1  # tokens 80 .. 95
    api.diffqkv_extend_window(step.q, step.cu, step.cache, 2, 4, 0.1, 200, out=out, dev_status=status)
    assert int(status.item()) == 0
    api.diffqkv_extend_window(step.q, step.cu, step.cache, 2, 4, 0.1, 206, out=out, dev_status=status)
    assert int(status.item()) == 1 << api.ERR_INDEX


def test_on_another_stream_and_two_at_once(api):
    steps = [forget(Step(api, [2000 + i, 50], [1 + i, 80], 16, 2, 4, 128, 128, seed=i).fill(), 500, 4) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in steps]
    outs = [torch.zeros((s.total_q, 16, 128), dtype=BF16, device="cuda") for s in steps]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, st, out in zip(steps, streams, outs):
            api.diffqkv_extend_window(s.q, s.cu, s.cache, 2, 4, 0.1, 500, sinks=4, out=out, stream=st)
    torch.cuda.synchronize()
    for s, out in zip(steps, outs):
        check(s, out, None, 0.1, 500, 4)


def test_a_captured_step_replays_with_other_lengths(api):
    steps = [Step(api, [1500, 3, 900, 0], n, 8, 2, 4, 64, 64, seed=3, room=300) for n in ([1, 1, 1, 1], [0, 200, 3, 60])]
    s = steps[0]
    cap = 300
    q = torch.zeros((cap, 8, 64), dtype=BF16, device="cuda")
    out = torch.full((cap, 8, 64), 77.0, dtype=BF16, device="cuda")
    pages = max(x.k.shape[0] for x in steps)
    k = torch.zeros((pages, 2, 16, 64), dtype=BF16, device="cuda")
    v = torch.zeros((pages, 4, 16, 64), dtype=BF16, device="cuda")
    row = max(x.table.shape[1] for x in steps)
    table = torch.zeros((4, row), dtype=torch.int32, device="cuda")
    lens, cu, status = ints([0] * 4), ints([0] * 5), ints([0])
    cache = api.KVCache(k, v, lens, row * 16, page_table=table, page_size=16)
    ws = torch.empty(api.diffqkv_extend_window_workspace_bytes(api.make_shape(4, 8, 2, 4, 64, 64, BF16, BF16, 1.0), cap),
                     dtype=torch.uint8, device="cuda")
    call = lambda: api.diffqkv_extend_window(q, cu, cache, 2, 4, 0.1, 250, sinks=20, out=out, workspace=ws,  # noqa: E731
                                             dev_status=status)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for s in steps + steps[:1]:
        s.fill()
        k[:s.k.shape[0]], v[:s.v.shape[0]] = s.k, s.v
        table.fill_(-1)
        table[:, :s.table.shape[1]] = s.table
        lens.copy_(s.lens)
        cu.copy_(s.cu)
        q[:s.total_q] = s.q
        out.fill_(77.0)
        graph.replay()
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        check(s, out, None, 0.1, 250, 20)
        assert bool((out[s.rows:] == 77.0).all())


@pytest.mark.parametrize("seed", range(24))
def test_random_steps(api, seed):
    r = random.Random(seed)
    n_q, n_k, n_v = HEADS[r.choice(list(HEADS))]
    dims = r.choice([(128, 128), (64, 64), (64, 128)])
    n = r.randint(1, 12)
    past = [r.choice([0, r.randint(0, 200), r.randint(0, 2500)]) for _ in range(n)]
    new = [r.choice([0, 1, 1, r.randint(1, 12), r.randint(1, 150)]) for _ in range(n)]
    window, sinks = r.choice([r.randint(1, 50), r.randint(1, 600), r.randint(1, 2000)]), r.choice([0, 0, 4, r.randint(0, 400)])
    step = Step(api, past, new, n_q, n_k, n_v, *dims, page=r.choice([8, 16, 32, 64, 128, 256]),
                layout=r.choice(["paged", "paged", "token", "flat"]), pad=r.randint(0, 3), seed=seed, room=r.randint(0, 50)).fill()
    run(api, forget(step, window, sinks), window, sinks)
