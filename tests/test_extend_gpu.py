"""diffqkv_extend: causal attention of ragged chunks over the cache, against the definition in float64."""
import math
import random

import pytest
import torch

from ragged import BF16, F32, Step, check_extend, ints

pytestmark = pytest.mark.gpu

HEADS = {"32/4/8": (32, 4, 8), "16/2/4": (16, 2, 4), "8/8/8": (8, 8, 8), "8/4/2": (8, 4, 2), "12/2/4": (12, 2, 4),
         "6/2/3": (6, 2, 3), "16/1/1": (16, 1, 1), "32/4/16": (32, 4, 16), "20/4/4": (20, 4, 4)}


@pytest.fixture(scope="module")
def api():
    from paper_2501_13629_b200 import api as _api
    return _api


def run(api, step, scale=None, out_dtype=None, want_lse=True, workspace=None):
    scale = step.d_qk ** -0.5 if scale is None else scale
    out = torch.full((step.total_q, step.n_q, step.d_v), 77.0, dtype=out_dtype or step.dtype, device="cuda")
    lse = torch.full((step.total_q, step.n_q), 77.0, dtype=F32, device="cuda") if want_lse else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.diffqkv_extend(step.q, step.cu, step.cache, step.n_k, step.n_v, scale, out=out, lse=lse, dev_status=status,
                       workspace=workspace)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    assert bool((out[step.rows:] == 77.0).all())  # rows behind the last chunk stay as they were
    if want_lse:
        assert bool((lse[step.rows:] == 77.0).all())
    check_extend(step, out, lse, scale)
    return out, lse


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dims", [(128, 128), (64, 64), (64, 128)])
def test_ragged_chunks_in_pages(api, heads, dims):
    """Chunks of every kind in one batch: none, one token, a few, around a tile, several tiles, with and without past."""
    past = [0, 5, 130, 127, 700, 0, 64, 1023, 300, 0]
    new = [1, 1, 4, 1, 33, 129, 0, 65, 257, 300]
    run(api, Step(api, past, new, *HEADS[heads], *dims, page=16, pad=3, seed=len(heads)).fill())


@pytest.mark.parametrize("page,layout", [(8, "paged"), (16, "token"), (32, "paged"), (64, "paged"), (128, "paged"),
                                         (256, "paged"), (16, "flat"), (24, "paged"), (4, "paged")])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_page_sizes_and_layouts(api, page, layout, dtype):
    """Pages that end inside a tile, tiles inside a page, token-major pools, no pages, and sizes only the plain kernel takes."""
    step = Step(api, [300, 0, 129, 17], [70, 140, 2, 1], 8, 2, 4, 128, 128, dtype=dtype, page=page, layout=layout,
                seed=page, room=40)
    run(api, step.fill())


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 383, 385, 512])
def test_single_sequence_lengths(api, length):
    """A whole prompt (no past), and the same length as past under a short chunk."""
    run(api, Step(api, [0], [length], 8, 2, 2, 128, 128, seed=length).fill())
    run(api, Step(api, [length], [3], 8, 2, 4, 128, 128, seed=length + 1, page=64).fill())


@pytest.mark.parametrize("past", [0, 1, 4000, 4095, 4096, 20000])
def test_one_long_row_is_split(api, past):
    """Few rows over a long cache: the token axis is divided over the SMs and joined."""
    run(api, Step(api, [past], [1], 32, 4, 8, 128, 128, seed=past).fill())
    run(api, Step(api, [past, 10], [5, 1], 32, 4, 16, 64, 64, seed=past + 1, page=64).fill())


@pytest.mark.parametrize("dtype,out_dtype", [(BF16, F32), (BF16, BF16), (F32, F32), (F32, BF16)])
def test_types(api, dtype, out_dtype):
    run(api, Step(api, [50, 400], [200, 3], 16, 2, 4, 64, 64, dtype=dtype, seed=3).fill(), out_dtype=out_dtype)


@pytest.mark.parametrize("dims", [(32, 32), (96, 80), (128, 256), (256, 128), (8, 512), (192, 128)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_other_head_dimensions(api, dims, dtype):
    run(api, Step(api, [33, 0, 200], [5, 40, 1], 4, 2, 4, *dims, dtype=dtype, seed=dims[0]).fill())


@pytest.mark.parametrize("scale", [-0.3, 0.0, 1.0])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scales(api, scale, dtype):
    run(api, Step(api, [33, 0, 200], [5, 40, 1], 4, 2, 4, 64, 64, dtype=dtype, seed=9, k_std=0.3).fill(), scale=scale)


def test_peaked_scores(api):
    """Keys ten times as large: the running maximum is raised often, most weights vanish."""
    run(api, Step(api, [900, 40], [140, 300], 8, 2, 4, 128, 128, seed=4, k_std=10.0).fill())


def test_rising_scores_raise_the_maximum_in_every_tile(api):
    step = Step(api, [1500], [130], 4, 1, 1, 128, 128, seed=5)
    ramp = torch.linspace(0.0, 12.0, 1630, device="cuda")
    step.q[:] = 1.0
    step.k_tok[0] = (ramp[:, None, None].expand(-1, 1, 128) / 4).to(BF16).contiguous()
    run(api, step.fill())


@pytest.mark.parametrize("choice", [1, 2])
@pytest.mark.parametrize("heads", ["32/4/8", "6/2/3", "16/1/1", "8/4/2"])
@pytest.mark.parametrize("dims", [(128, 128), (64, 64), (64, 128), (128, 64)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_kernels_on_fmas(api, choice, heads, dims, dtype):
    """The kernels that take what the tensor cores do not, on the same steps: many rows, and few over a long cache."""
    api.extend_kernel(choice)
    try:
        run(api, Step(api, [0, 5, 130, 700, 0], [1, 4, 33, 129, 0], *HEADS[heads], *dims, dtype=dtype, seed=21).fill())
        assert api.last_extend_kernel() == choice
        run(api, Step(api, [3000, 90, 1024], [2, 1, 1], *HEADS[heads], *dims, dtype=dtype, seed=22, pad=2).fill())
    finally:
        api.extend_kernel(0)


def test_which_kernel(api):
    for kw, kernel in ((dict(), 3), (dict(dtype=F32), 2), (dict(page=24), 2), (dict(page=64), 3), (dict(layout="flat"), 3)):
        run(api, Step(api, [30, 9], [5, 40], 8, 2, 4, 64, 64, seed=23, **kw).fill())
        assert api.last_extend_kernel() == kernel, kw
    run(api, Step(api, [30, 9], [5, 40], 8, 2, 4, 64, 64, seed=23).fill(), scale=-0.1)
    assert api.last_extend_kernel() == 2
    run(api, Step(api, [30, 9], [5, 40], 8, 2, 4, 96, 64, seed=23).fill())
    assert api.last_extend_kernel() == 1


def test_nothing_to_do(api):
    step = Step(api, [3, 9], [0, 0], 4, 2, 2, 64, 64, pad=5).fill()
    run(api, step)
    out = api.diffqkv_extend(step.q[:0], step.cu, step.cache, 2, 2, 0.1)
    assert out.shape == (0, 4, 64)


def test_many_sequences(api):
    """More sequences than a block has threads, most of them with a token or none."""
    r = random.Random(1)
    past = [r.randint(0, 90) for _ in range(700)]
    new = [r.choice([0, 1, 1, 1, 2, 7]) for _ in range(700)]
    run(api, Step(api, past, new, 8, 2, 4, 64, 64, seed=6).fill())


def test_many_sequences_of_both_kinds(api):
    """Several sequences to a thread in both lists, sequences of either kind anywhere among the others."""
    r = random.Random(2)
    past = [r.randint(0, 60) for _ in range(1900)]
    new = [r.choice([0, 1, 1, 2, 3, 40, 130]) if i % 5 == 0 else r.choice([0, 0, 1]) for i in range(1900)]
    run(api, Step(api, past, new, 8, 2, 4, 64, 64, seed=9, pad=3).fill())


@pytest.mark.parametrize("heads", ["32/4/8", "16/2/4", "6/2/3", "16/1/1", "32/4/16"])
@pytest.mark.parametrize("load", ["one chunk", "one token", "even", "short caches"])
def test_long_chunks_beside_single_rows(api, heads, load):
    """The two kinds divide the SMs: nearly all of the work of one kind, of the other, of both, and too little for all."""
    past, new = {"one chunk": ([2000] + [3] * 2, [600] + [1] * 2), "one token": ([20] + [4000] * 12, [70] + [2] * 12),
                 "even": ([900, 1500] + [2500] * 10, [200, 100] + [1, 2, 3, 1, 1] * 2),
                 "short caches": ([0, 1, 2, 3], [65, 1, 1, 66])}[load]
    run(api, Step(api, past, new, *HEADS[heads], 128, 128, seed=len(load), pad=2).fill())


@pytest.mark.parametrize("dtype,dims", [(BF16, (128, 128)), (BF16, (64, 64)), (F32, (64, 64)), (F32, (96, 80))])
@pytest.mark.parametrize("past", [40, 500, 9000])
def test_a_row_that_is_not_finite_stays_alone(api, dtype, dims, past):
    """NaN and infinity in one query row reach its own results, all of them, in chunks of either kind."""
    for new, bad in (([3, 2], 1), ([200, 3], 77), ([200, 3], 201)):
        step = Step(api, [past, 40], new, 8, 2, 4, *dims, dtype=dtype, seed=11).fill()
        clean, clean_lse = run(api, step)
        for x in (math.nan, math.inf):
            q = step.q.clone()
            q[bad, 3] = x
            lse = torch.empty_like(clean_lse)
            out = api.diffqkv_extend(q, step.cu, step.cache, 2, 4, step.d_qk ** -0.5, lse=lse)
            torch.cuda.synchronize()
            assert not bool(torch.isfinite(out[bad, 3]).any()) and bool(lse[bad, 3].isnan())
            out[bad, 3], lse[bad, 3] = clean[bad, 3], clean_lse[bad, 3]
            assert torch.equal(out, clean) and torch.equal(lse, clean_lse)


@pytest.mark.parametrize("seed", range(12))
def test_random_steps(api, seed):
    r = random.Random(seed)
    heads = r.choice(list(HEADS.values()))
    dims = r.choice([(128, 128), (64, 64), (64, 128)])
    B = r.randint(1, 9)
    past = [r.choice([0, r.randint(0, 200), r.randint(0, 3000)]) for _ in range(B)]
    new = [r.choice([0, 1, r.randint(1, 9), r.randint(1, 400)]) for _ in range(B)]
    if sum(new) == 0:
        new[0] = 1
    run(api, Step(api, past, new, *heads, *dims, page=r.choice([8, 16, 32, 64, 128, 256]), seed=seed + 100,
                  layout=r.choice(["paged", "token", "flat"]), pad=r.randint(0, 4), room=r.randint(0, 300)).fill())


def test_results_do_not_depend_on_the_call(api):
    """Two calls give the same bits; a workspace full of NaN changes nothing; another stream neither."""
    step = Step(api, [3000, 12, 700], [3, 90, 300], 16, 2, 4, 128, 128, seed=8).fill()
    first, lse = run(api, step)
    shape = api.make_shape(3, 16, 2, 4, 128, 128, BF16, BF16, 1.0)
    ws = torch.full((api.diffqkv_extend_workspace_bytes(shape, step.total_q),), 255, dtype=torch.uint8, device="cuda")
    again, lse2 = run(api, step, workspace=ws)
    assert torch.equal(first, again) and torch.equal(lse, lse2)
    side = torch.cuda.Stream()
    out = torch.empty_like(first)
    side.wait_stream(torch.cuda.current_stream())
    api.diffqkv_extend(step.q, step.cu, step.cache, 2, 4, 128 ** -0.5, out=out, workspace=ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(out, first)


def test_matches_decode_and_prefill(api):
    """A chunk of one is diffqkv_decode; equal chunks are diffqkv_prefill."""
    step = Step(api, [100, 900], [1, 1], 16, 2, 4, 128, 128, seed=11).fill()
    out, lse = run(api, step, out_dtype=F32)
    counted = api.KVCache(step.k, step.v, step.lens + 1, step.max_seqlen, page_table=step.table, page_size=16)
    ref = api.diffqkv_decode(step.q, counted, 2, 4, 128 ** -0.5, out_dtype=F32)
    assert float((out - ref).abs().max()) <= 2 * 2.0 ** -8 * float(step.v_tok[0].float().abs().max())
    step = Step(api, [100, 900], [200, 200], 16, 2, 4, 128, 128, seed=12).fill()
    out, _ = run(api, step, out_dtype=F32)
    k_new = torch.stack([k[p:] for k, p in zip(step.k_tok, step.past)])
    v_new = torch.stack([v[p:] for v, p in zip(step.v_tok, step.past)])
    ref = api.diffqkv_prefill(step.q.view(2, 200, 16, 128), k_new, v_new, step.cache, 128 ** -0.5, out_dtype=F32)
    assert float((out.view_as(ref) - ref).abs().max()) <= 2 * 2.0 ** -8 * 6


def test_replayed_with_other_lengths(api):
    """A captured step is replayed after the lengths and the chunks have changed in place."""
    step = Step(api, [40, 700, 0], [30, 1, 99], 8, 2, 4, 128, 128, seed=13, room=300, pad=70).fill()
    other = Step(api, [10, 200, 129], [150, 50, 0], 8, 2, 4, 128, 128, seed=14, room=300)
    assert other.total_q == step.total_q
    other.fill()
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    out = torch.zeros((step.total_q, 8, 128), dtype=BF16, device="cuda")
    pages = max(step.k.shape[0], other.k.shape[0])
    k, v = (torch.zeros((pages,) + tuple(x.shape[1:]), dtype=BF16, device="cuda") for x in (step.k, step.v))
    row = max(step.table.shape[1], other.table.shape[1])
    table = torch.zeros((3, row), dtype=torch.int32, device="cuda")
    lens, cu, q = torch.zeros(3, dtype=torch.int32, device="cuda"), ints([0, 0, 0, 0]), torch.zeros_like(step.q)
    cache = api.KVCache(k, v, lens, row * 16, page_table=table, page_size=16)
    call = lambda: api.diffqkv_extend(q, cu, cache, 2, 4, 128 ** -0.5, out=out, workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for s in (step, other, step):
        k[:s.k.shape[0]], v[:s.v.shape[0]] = s.k, s.v
        table[:, :s.table.shape[1]] = s.table
        lens.copy_(s.lens), cu.copy_(s.cu), q.copy_(s.q)
        graph.replay()
        torch.cuda.synchronize()
        check_extend(s, out, None, 128 ** -0.5)


def test_sequences_that_do_not_fit_are_skipped(api):
    """past + n beyond the cache, a negative length and a cu_q out of order: reported, their rows stay, others are right."""
    step = Step(api, [40, 16, 20], [30, 1, 9], 8, 2, 4, 64, 64, seed=15).fill()
    out = torch.full((40, 8, 64), 7.0, dtype=BF16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for lens in ([step.max_seqlen - 29, 16, 20], [-1, 16, 20]):
        out.fill_(7.0)
        status.zero_()
        cache = api.KVCache(step.k, step.v, ints(lens), step.max_seqlen, page_table=step.table, page_size=16)
        api.diffqkv_extend(step.q, step.cu, cache, 2, 4, 0.125, out=out, dev_status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == 1 << api.ERR_INDEX
        assert bool((out[:30] == 7.0).all())
        kept = Step.__new__(Step)
        kept.__dict__.update(step.__dict__)
        kept.new = [0, 1, 9]
        check_extend(kept, out, None, 0.125)
    for cu in ([0, 30, 29, 40], [0, 30, 31, 41], [0, -5, 31, 40]):
        status.zero_()
        api.diffqkv_extend(step.q, ints(cu), step.cache, 2, 4, 0.125, out=out, dev_status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == 1 << api.ERR_INDEX


@pytest.mark.parametrize("bad", [-1, 10 ** 6])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_bad_page_ids_are_reported(api, bad, dtype):
    step = Step(api, [40, 16], [30, 1], 8, 2, 4, 64, 64, dtype=dtype, seed=16).fill()
    step.table[0, 1] = bad
    out = torch.zeros((31, 8, 64), dtype=dtype, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.diffqkv_extend(step.q, step.cu, step.cache, 2, 4, 0.125, out=out, dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 1 << api.ERR_INDEX
    kept = Step.__new__(Step)
    kept.__dict__.update(step.__dict__)
    kept.new = [0, 1]
    check_extend(kept, out, None, 0.125)


def test_offsets_beyond_32_bits(api):
    """Pages whose element offsets pass 2^31 (and byte offsets 2^32): a pool of 5 GB of which two ends are used."""
    pages, page, n_k, n_v, d = 40000, 128, 2, 2, 128
    k = torch.zeros((pages, n_k, page, d), dtype=BF16, device="cuda")
    v = torch.zeros((pages, n_v, page, d), dtype=BF16, device="cuda")
    step = Step(api, [200], [3], 4, n_k, n_v, d, d, page=page, seed=17)
    assert k.numel() > 1 << 30 and (pages - 1) * k.stride(0) * 2 > 1 << 31
    step.k, step.v = k, v
    step.table = ints([[pages - 1, 0]])
    step.cache = api.KVCache(k, v, step.lens, 256, page_table=step.table, page_size=page)
    run(api, step.fill())
