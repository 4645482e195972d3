"""diffqkv_extend_shared: sequences that share a prefix, against the definition in float64."""
import math
import random

import pytest
import torch

from ragged import BF16, F32, Step, ints
from ranged import check

pytestmark = pytest.mark.gpu

HEADS = {"32/4/8": (32, 4, 8), "16/2/4": (16, 2, 4), "8/8/8": (8, 8, 8), "8/4/2": (8, 4, 2), "12/2/4": (12, 2, 4),
         "6/2/3": (6, 2, 3), "16/1/1": (16, 1, 1), "32/4/16": (32, 4, 16), "20/4/4": (20, 4, 4)}


@pytest.fixture(scope="module")
def api():
    from paper_2501_13629_b200 import api as _api
    return _api


def share(step, groups, prefix, same_pages=True):
    """The sequences of every group get the first one's first tokens, in the same pages where those are whole."""
    step.fill()
    for g, p in enumerate(prefix):
        for b in range(groups[g] + 1, groups[g + 1]):
            a = groups[g]
            if not 0 < p <= min(step.total[a], step.total[b]):
                continue
            step.k_tok[b][:p], step.v_tok[b][:p] = step.k_tok[a][:p], step.v_tok[a][:p]
            blk, slot = step.place(b, 0, p)
            step.k[blk, :, slot], step.v[blk, :, slot] = step.k_tok[b][:p], step.v_tok[b][:p]
            if same_pages and step.table is not None:
                step.table[b, :p // step.page] = step.table[a, :p // step.page]
    return step


def run(api, step, groups, prefix, scale=None, out_dtype=None, want_lse=True, workspace=None):
    scale = step.d_qk ** -0.5 if scale is None else scale
    out = torch.full((step.total_q, step.n_q, step.d_v), 77.0, dtype=out_dtype or step.dtype, device="cuda")
    lse = torch.full((step.total_q, step.n_q), 77.0, dtype=F32, device="cuda") if want_lse else None
    status = ints([0])
    api.diffqkv_extend_shared(step.q, step.cu, step.cache, ints(groups), ints(prefix), step.n_k, step.n_v, scale, out=out,
                              lse=lse, dev_status=status, workspace=workspace)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    assert bool((out[step.rows:] == 77.0).all())  # rows behind the last chunk stay as they were
    if want_lse:
        assert bool((lse[step.rows:] == 77.0).all())
    check(step, out, lse, scale, joined=True)
    return out, lse


# outside of the groups, a pair, a group whose first sequence has no rows, one that shares nothing, one sequence alone, none
PAST = [40, 300, 517, 260, 260, 290, 10, 700, 129, 0]
NEW = [3, 1, 1, 0, 40, 130, 2, 1, 5, 70]
GROUPS, PREFIX = [1, 3, 6, 6, 8, 9], [299, 256, 50, 0, 128]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dims", [(128, 128), (64, 64), (64, 128)])
def test_groups_of_every_kind(api, heads, dims):
    step = Step(api, PAST, NEW, *HEADS[heads], *dims, page=16, pad=3, seed=len(heads))
    run(api, share(step, GROUPS, PREFIX), GROUPS, PREFIX)


@pytest.mark.parametrize("prefix", [1, 15, 16, 17, 127, 128, 129, 255, 256, 640, 1500])
@pytest.mark.parametrize("new", [[1, 1, 1], [1, 9, 200], [64, 64, 64]])
def test_prefix_lengths(api, prefix, new):
    """Prefixes that end in a page, at its end, in a tile, at its end; rows right behind them."""
    step = Step(api, [prefix, prefix + 1, prefix + 130], new, 16, 2, 4, 128, 128, page=16, seed=prefix)
    run(api, share(step, [0, 3], [prefix]), [0, 3], [prefix])


@pytest.mark.parametrize("batch", [2, 9, 33, 64, 200])
def test_many_sequences_behind_one_prefix(api, batch):
    r = random.Random(batch)
    past = [1000 + r.randint(0, 90) for _ in range(batch)]
    step = Step(api, past, [1] * batch, 8, 2, 4, 64, 64, page=32, seed=batch)
    run(api, share(step, [0, batch], [1000]), [0, batch], [1000])


@pytest.mark.parametrize("groups", [1, 7, 40])
def test_many_groups(api, groups):
    r = random.Random(groups)
    ends, prefix, past = [0], [], []
    for _ in range(groups):
        n, p = r.randint(1, 9), r.randint(0, 400)
        past += [p + r.randint(0, 60) for _ in range(n)]
        ends.append(ends[-1] + n)
        prefix.append(p)
    new = [r.choice([0, 1, 1, 2, r.randint(1, 30)]) for _ in past]
    step = Step(api, past, new, 16, 2, 4, 64, 128, page=16, seed=groups, pad=2)
    run(api, share(step, ends, prefix), ends, prefix)


@pytest.mark.parametrize("page,layout", [(8, "paged"), (16, "token"), (32, "paged"), (64, "paged"), (128, "paged"),
                                         (256, "paged"), (16, "flat"), (24, "paged"), (4, "paged")])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_page_sizes_and_layouts(api, page, layout, dtype):
    step = Step(api, [300, 333, 129, 130, 17], [1, 40, 2, 1, 30], 8, 2, 4, 128, 128, dtype=dtype, page=page, layout=layout,
                seed=page, room=40)
    run(api, share(step, [0, 2, 4], [300, 70]), [0, 2, 4], [300, 70])


@pytest.mark.parametrize("dtype,out_dtype", [(BF16, F32), (BF16, BF16), (F32, F32), (F32, BF16)])
def test_types(api, dtype, out_dtype):
    step = Step(api, [200, 400], [200, 3], 16, 2, 4, 64, 64, dtype=dtype, seed=3)
    run(api, share(step, [0, 2], [190]), [0, 2], [190], out_dtype=out_dtype, want_lse=out_dtype == F32)


@pytest.mark.parametrize("dims", [(32, 32), (96, 80), (128, 256), (128, 64)])
def test_other_head_dimensions(api, dims):
    step = Step(api, [133, 150, 20], [5, 40, 1], 4, 2, 4, *dims, seed=dims[0])
    run(api, share(step, [0, 2], [100]), [0, 2], [100])


@pytest.mark.parametrize("heads", ["32/4/8", "6/2/3", "8/8/8", "16/1/1", "12/2/4"])
@pytest.mark.parametrize("new", [[5, 5, 6], [16, 17, 1], [10, 11, 22], [33, 31, 64], [60, 65, 4], [1, 128, 130]])
@pytest.mark.parametrize("prefix", [20, 150])
def test_rows_around_what_is_few(api, heads, new, prefix):
    """Rows of groups and of sequences that fill the blocks of the kernel of few rows, one less and one more."""
    step = Step(api, [prefix + 7 * i for i in range(3)] + [40], new + [18], *HEADS[heads], 64, 128, page=32, seed=sum(new), pad=2)
    run(api, share(step, [0, 3], [prefix]), [0, 3], [prefix])


def test_a_shared_prefix_is_read_once(api):
    """From the first sequence: what the others have in its place does not matter here."""
    step = Step(api, [500, 520, 600, 77], [1, 9, 2, 3], 16, 2, 4, 128, 128, seed=3)
    share(step, [0, 3], [430], same_pages=False)
    for b in (1, 2):
        blk, slot = step.place(b, 0, 430)
        step.k[blk, :, slot] = math.nan
        step.v[blk, :, slot] = math.nan
        step.table[b, :430 // 16] = -1
    run(api, step, [0, 3], [430])
    assert api.last_extend_kernel() == 3


@pytest.mark.parametrize("k_std", [10.0, 40.0])
def test_peaked_scores(api, k_std):
    """One of the two parts has nearly all of the weight."""
    step = Step(api, [900, 940, 905], [3, 140, 1], 8, 2, 4, 128, 128, seed=4, k_std=k_std)
    run(api, share(step, [0, 3], [890]), [0, 3], [890])


@pytest.mark.parametrize("new", [1, 90])
@pytest.mark.parametrize("where", ["prefix", "own", "both"])
def test_parts_of_minus_infinity(api, new, where):
    step = Step(api, [300, 310], [new, new], 4, 2, 2, 64, 64, seed=2)
    step.q[:] = step.q.abs() + 0.1
    for b in range(2):
        if where != "own":
            step.k_tok[b][:256] = -math.inf
        if where != "prefix":
            step.k_tok[b][256:] = -math.inf
    share(step, [0, 2], [256])
    out, lse = torch.empty((2 * new, 4, 64), dtype=F32, device="cuda"), torch.empty((2 * new, 4), dtype=F32, device="cuda")
    api.diffqkv_extend_shared(step.q, step.cu, step.cache, ints([0, 2]), ints([256]), 2, 2, 0.125, out=out, lse=lse)
    if where == "both":
        assert bool((out == 0).all()) and bool((lse == -math.inf).all())
        return
    plain, plain_lse = torch.empty_like(out), torch.empty_like(lse)
    api.diffqkv_extend(step.q, step.cu, step.cache, 2, 2, 0.125, out=plain, lse=plain_lse)
    assert bool(torch.isfinite(out).all()) and bool(((lse - plain_lse).abs() <= 1e-5).all())
    assert bool(((out - plain).abs() <= 2 ** -7 * 5).all())  # weights of bf16 in either, values up to 5


def test_nan_stays_with_its_sequences(api):
    step = Step(api, [300, 310, 200, 200], [2, 30, 1, 1], 4, 2, 2, 128, 128, seed=2)
    share(step, [0, 2, 4], [256, 100])
    out = torch.empty((34, 4, 128), dtype=BF16, device="cuda")
    blk, slot = step.place(2, 150, 151)  # own token of the third
    step.k[blk, :, slot] = math.nan
    blk, slot = step.place(0, 10, 11)    # of the first group's prefix
    step.k[blk, :, slot] = math.nan
    api.diffqkv_extend_shared(step.q, step.cu, step.cache, ints([0, 2, 4]), ints([256, 100]), 2, 2, 0.1, out=out)
    assert bool(torch.isnan(out[:33]).all()) and bool(torch.isfinite(out[33]).all())


def test_repeats_bit_for_bit_and_with_any_workspace(api):
    step = share(Step(api, PAST, NEW, 32, 4, 8, 128, 128, seed=5), GROUPS, PREFIX)
    first, lse = run(api, step, GROUPS, PREFIX)
    nbytes = api.diffqkv_extend_shared_workspace_bytes(api.make_shape(10, 32, 4, 8, 128, 128, BF16, BF16, 1.0), step.total_q)
    for fill in (0, 255):
        ws = torch.full((nbytes,), fill, dtype=torch.uint8, device="cuda")
        again, lse2 = run(api, step, GROUPS, PREFIX, workspace=ws)
        assert torch.equal(first, again) and torch.equal(lse, lse2)


def test_no_groups_is_extend(api):
    step = Step(api, PAST, NEW, 16, 2, 4, 128, 128, seed=8, pad=2).fill()
    out = torch.empty((step.total_q, 16, 128), dtype=BF16, device="cuda")
    api.diffqkv_extend(step.q, step.cu, step.cache, 2, 4, 0.1, out=out)
    got, _ = run(api, step, [0], [], scale=0.1)
    assert torch.equal(got[:step.rows], out[:step.rows])
    got, _ = run(api, step, [0, 4, 10], [0, 0], scale=0.1)  # groups that share nothing
    assert bool(((got[:step.rows] - out[:step.rows]).abs() <= 2 ** -6).all())


@pytest.mark.parametrize("dtype,dims", [(BF16, (128, 128)), (F32, (64, 64)), (BF16, (96, 80))])
def test_sequences_that_do_not_fit(api, dtype, dims):
    """Reported and skipped; the others are as they would be."""
    def call(groups, prefix, lens=None, bad=()):
        step = Step(api, [300, 310, 290, 50, 40], [3, 40, 1, 1, 20], 8, 2, 4, *dims, dtype=dtype, seed=7, pad=1)
        share(step, [0, 3, 5], [200, 45])
        if lens:
            step.lens.copy_(ints(lens))
        out = torch.full((step.total_q, 8, dims[1]), 77.0, dtype=dtype, device="cuda")
        status = ints([0])
        api.diffqkv_extend_shared(step.q, step.cu, step.cache, ints(groups), ints(prefix), 2, 4, 0.1, out=out, dev_status=status)
        assert int(status.item()) == (1 << api.ERR_INDEX if bad else 0)
        for b in bad:
            assert bool((out[step.cu_host[b]:step.cu_host[b + 1]] == 77.0).all()), b
        assert bool((out[step.rows:] == 77.0).all())
        check(step, out, None, 0.1, joined=True, only=[b for b in range(5) if b not in bad])

    call([0, 3], [200])
    call([0, 3], [200], lens=[300, -1, 290, 50, 40], bad=[1])           # a denied sequence
    call([0, 3, 5], [200, 40])
    call([0, 3, 5], [200, 45], bad=[4])                                 # a prefix longer than the cache of one
    call([0, 3, 5], [200, -1], bad=[3, 4])
    call([0, 3, 9], [200, 0], bad=[3, 4])                               # a group that ends outside of the batch
    call([-1, 3], [200], bad=[0, 1, 2])
    call([0, 3, 5], [200, 1 << 30], bad=[3, 4])


@pytest.mark.parametrize("bad", [None, 0, 2])
def test_a_few_rows_in_all(api, bad):
    """Steps that one kernel takes alone, with a sequence that does not fit among them."""
    step = Step(api, [300, 310, 290, 50], [1, 0, 2, 1], 8, 2, 4, 128, 128, seed=7, pad=2)
    share(step, [0, 3], [200])
    if bad is not None:
        step.lens[bad] = -1 if bad else 199
    out, status = torch.full((step.total_q, 8, 128), 77.0, dtype=BF16, device="cuda"), ints([0])
    api.diffqkv_extend_shared(step.q, step.cu, step.cache, ints([0, 3]), ints([200]), 2, 4, 0.1, out=out, dev_status=status)
    assert int(status.item()) == (0 if bad is None else 1 << api.ERR_INDEX)
    check(step, out, None, 0.1, joined=True, only=[b for b in range(4) if b != bad])
    if bad is not None:
        assert bool((out[step.cu_host[bad]:step.cu_host[bad + 1]] == 77.0).all())
    assert bool((out[step.rows:] == 77.0).all())


@pytest.mark.parametrize("groups,size", [(450, 2), (3, 300)])
def test_more_entries_than_threads(api, groups, size):
    r = random.Random(groups)
    ends, prefix, past = [0], [], []
    for _ in range(groups):
        p = r.randint(0, 90)
        past += [p + r.randint(0, 60) for _ in range(size)]
        ends.append(ends[-1] + size)
        prefix.append(p)
    new = [r.choice([0, 1, 1, 2, 30]) for _ in past]
    step = Step(api, past, new, 8, 2, 4, 64, 64, page=16, seed=groups, pad=2)
    run(api, share(step, ends, prefix), ends, prefix)


def test_groups_that_go_back(api):
    """cu_seqs decreases, so that groups of rows overlap: reported, and the step is left out."""
    step = Step(api, [300, 310, 290, 305, 20, 40], [3, 4, 2, 1, 5, 60], 8, 2, 4, 128, 128, seed=7, pad=4)
    share(step, [0, 4], [200])
    nbytes = api.diffqkv_extend_shared_workspace_bytes(api.make_shape(6, 8, 2, 4, 128, 128, BF16, BF16, 0.1), step.total_q)
    ws = torch.zeros(nbytes, dtype=torch.uint8, device="cuda")
    for groups, back in (([0, 4, 4, 4], False), ([0, 4, 2, 4], True), ([2, 4, 0, 4], True), ([0, 4, 4, 6], False)):
        out, status = torch.full((step.total_q, 8, 128), 77.0, dtype=BF16, device="cuda"), ints([0])
        api.diffqkv_extend_shared(step.q, step.cu, step.cache, ints(groups), ints([200, 200, 0]), 2, 4, 0.1, out=out,
                                  workspace=ws, dev_status=status)
        assert int(status.item()) == (1 << api.ERR_INDEX if back else 0)
        if back:
            assert bool((out == 77.0).all())
        else:
            check(step, out, None, 0.1, joined=True)
        assert bool((out[step.rows:] == 77.0).all())


def test_rows_out_of_order_are_not_written(api):
    """cu_q decreases inside a group: its sequences' rows are not the group's."""
    step = Step(api, [300, 310, 290], [3, 4, 2], 8, 2, 4, 128, 128, seed=7, pad=4)
    share(step, [0, 3], [200])
    out, status = torch.full((step.total_q, 8, 128), 77.0, dtype=BF16, device="cuda"), ints([0])
    api.diffqkv_extend_shared(step.q, ints([0, 3, 12, 9]), step.cache, ints([0, 3]), ints([200]), 2, 4, 0.1, out=out,
                              dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 1 << api.ERR_INDEX
    assert bool((out[9:] == 77.0).all())


def test_two_calls_at_once_and_other_streams(api):
    steps = [share(Step(api, [2000 + i, 2050], [1 + i, 80], 16, 2, 4, 128, 128, seed=i), [0, 2], [1999]) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in steps]
    outs = [torch.zeros((s.total_q, 16, 128), dtype=BF16, device="cuda") for s in steps]
    cu, lens = ints([0, 2]), ints([1999])
    torch.cuda.synchronize()
    for _ in range(20):
        for s, st, out in zip(steps, streams, outs):
            api.diffqkv_extend_shared(s.q, s.cu, s.cache, cu, lens, 2, 4, 0.1, out=out, stream=st)
    torch.cuda.synchronize()
    for s, out in zip(steps, outs):
        check(s, out, None, 0.1, joined=True)


def test_a_captured_step_replays_with_other_groups(api):
    cap = 120
    variants = [([300, 310, 290, 500], [1, 1, 1, 1], [0, 3, 3], [256, 0]), ([300, 310, 500, 505], [0, 40, 1, 30], [0, 2, 4], [77, 500]),
                ([0, 5, 10, 0], [3, 1, 1, 40], [1, 1, 1], [0, 0])]
    q = torch.zeros((cap, 8, 64), dtype=BF16, device="cuda")
    out = torch.full((cap, 8, 64), 77.0, dtype=BF16, device="cuda")
    steps = [share(Step(api, p, n, 8, 2, 4, 64, 64, seed=3, room=60), g, l) for p, n, g, l in variants]
    pages, row = max(s.k.shape[0] for s in steps), max(s.table.shape[1] for s in steps)
    k = torch.zeros((pages, 2, 16, 64), dtype=BF16, device="cuda")
    v = torch.zeros((pages, 4, 16, 64), dtype=BF16, device="cuda")
    table = torch.zeros((4, row), dtype=torch.int32, device="cuda")
    lens, cu, status, groups, prefix = ints([0] * 4), ints([0] * 5), ints([0]), ints([0, 0, 0]), ints([0, 0])
    cache = api.KVCache(k, v, lens, row * 16, page_table=table, page_size=16)
    nbytes = api.diffqkv_extend_shared_workspace_bytes(api.make_shape(4, 8, 2, 4, 64, 64, BF16, BF16, 1.0), cap)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    call = lambda: api.diffqkv_extend_shared(q, cu, cache, groups, prefix, 2, 4, 0.1, out=out, workspace=ws,  # noqa: E731
                                             dev_status=status)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in (0, 1, 2, 0):
        s, (_, _, g, l) = steps[i], variants[i]
        k[:s.k.shape[0]], v[:s.v.shape[0]] = s.k, s.v
        table.fill_(-1)
        table[:, :s.table.shape[1]] = s.table
        lens.copy_(s.lens)
        cu.copy_(s.cu)
        groups.copy_(ints(g))
        prefix.copy_(ints(l))
        q[:s.total_q] = s.q
        out.fill_(77.0)
        graph.replay()
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        check(s, out, None, 0.1, joined=True)
        assert bool((out[s.rows:] == 77.0).all())


@pytest.mark.parametrize("seed", range(24))
def test_random_steps(api, seed):
    r = random.Random(seed)
    n_q, n_k, n_v = HEADS[r.choice(list(HEADS))]
    dims = r.choice([(128, 128), (64, 64), (64, 128)])
    n = r.randint(1, 12)
    ends = sorted(r.randint(0, n) for _ in range(r.randint(2, 5)))
    prefix = [r.choice([0, r.randint(1, 300), r.randint(1, 2000)]) for _ in ends[1:]]
    past = [r.randint(0, 300) for _ in range(n)]
    for g, p in enumerate(prefix):
        for b in range(ends[g], ends[g + 1]):
            past[b] = p + r.choice([0, r.randint(0, 200)])
    new = [r.choice([0, 1, 1, r.randint(1, 12), r.randint(1, 150)]) for _ in range(n)]
    step = Step(api, past, new, n_q, n_k, n_v, *dims, page=r.choice([8, 16, 32, 64, 128, 256]),
                layout=r.choice(["paged", "paged", "token", "flat"]), pad=r.randint(0, 3), seed=seed, room=r.randint(0, 50))
    run(api, share(step, ends, prefix), ends, prefix)


@pytest.mark.parametrize("layout", ["paged", "flat"])
@pytest.mark.parametrize("first", [0, 5999, -1])
@pytest.mark.parametrize("new", [[0, 1, 2], [0, 3, 120], [2, 1, 2], [3, 1, 90]])
def test_a_first_sequence_without_the_prefix(api, layout, first, new):
    """What it has behind its length are not the group's tokens: the others read their own."""
    step = Step(api, [6000, 6100, 6050, 90], new + [5], 16, 2, 4, 128, 128, layout=layout, seed=sum(new), pad=2)
    share(step, [0, 3], [6000], same_pages=False)
    blk, slot = step.place(0, max(first, 0), 6000)
    step.k[blk, :, slot] = 0.5  # left there by somebody else
    step.v[blk, :, slot] = -3.0
    if layout == "paged":
        step.table[0, -(-max(first, 0) // step.page):] = -1
    step.lens[0] = first
    out, status = torch.full((step.total_q, 16, 128), 77.0, dtype=BF16, device="cuda"), ints([0])
    api.diffqkv_extend_shared(step.q, step.cu, step.cache, ints([0, 3]), ints([6000]), 2, 4, 0.1, out=out, dev_status=status)
    fits = first >= 0 and new[0] == 0  # (a length below 0 is reported of a sequence without rows too)
    assert int(status.item()) == (0 if fits else 1 << api.ERR_INDEX)
    check(step, out, None, 0.1, joined=True, only=[1, 2, 3])
    assert bool((out[:new[0]] == 77.0).all()) and bool((out[step.rows:] == 77.0).all())
