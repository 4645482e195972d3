"""diffqkv_extend_shared with every prefix read once that can be, whatever that saves: from the first sequence of its group, in
either of the two kernels, whole and cut, and joined with the rows' own parts."""
import math
import random

import pytest
import torch

from ragged import BF16, F32, HALF_STEP, Step, ints
from ranged import attend64, check, visible
from test_extend_shared_gpu import GROUPS, HEADS, NEW, PAST, PREFIX, run, share

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2501_13629_b200 import api as _api
    return _api


@pytest.fixture(autouse=True)
def always(api):
    api.extend_sharing(1)
    yield
    api.extend_sharing(0)


def hide(step, groups, prefix):
    """Only the first sequence of a group has its prefix: the others' own copies become NaN, their whole pages are taken away."""
    share(step, groups, prefix, same_pages=False)
    for g, p in enumerate(prefix):
        for b in range(groups[g] + 1, groups[g + 1]):
            if 0 < p <= step.total[b]:
                blk, slot = step.place(b, 0, p)
                step.k[blk, :, slot] = math.nan
                step.v[blk, :, slot] = math.nan
                if step.table is not None:
                    step.table[b, :p // step.page] = -1
    return step


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dims", [(128, 128), (64, 64), (64, 128)])
def test_groups_of_every_kind(api, heads, dims):
    step = Step(api, PAST, NEW, *HEADS[heads], *dims, page=16, pad=3, seed=len(heads))
    run(api, hide(step, GROUPS, PREFIX), GROUPS, PREFIX)
    assert api.last_extend_kernel() == 3


@pytest.mark.parametrize("prefix", [1, 15, 16, 17, 127, 128, 129, 255, 256, 640, 1500])
@pytest.mark.parametrize("new", [[1, 1, 1], [1, 9, 200], [64, 64, 64], [300, 2, 700]])
def test_prefix_lengths(api, prefix, new):
    step = Step(api, [prefix, prefix + 1, prefix + 130], new, 16, 2, 4, 128, 128, page=16, seed=prefix)
    run(api, hide(step, [0, 3], [prefix]), [0, 3], [prefix])


@pytest.mark.parametrize("page,layout", [(8, "paged"), (16, "token"), (32, "paged"), (64, "paged"), (128, "paged"),
                                         (256, "paged"), (16, "flat")])
@pytest.mark.parametrize("heads", ["8/4/2", "8/8/8"])
def test_page_sizes_and_layouts(api, page, layout, heads):
    step = Step(api, [300, 333, 129, 130, 17], [1, 240, 2, 1, 30], *HEADS[heads], 128, 128, page=page, layout=layout, seed=page,
                room=40)
    run(api, hide(step, [0, 2, 4], [300, 70]), [0, 2, 4], [300, 70])


@pytest.mark.parametrize("out_dtype", [BF16, F32])
@pytest.mark.parametrize("new", [[200, 3], [2, 1]])
def test_types(api, out_dtype, new):
    step = Step(api, [200, 400], new, 16, 2, 4, 64, 64, seed=3)
    run(api, hide(step, [0, 2], [190]), [0, 2], [190], out_dtype=out_dtype, want_lse=out_dtype == F32)


@pytest.mark.parametrize("heads", ["32/4/8", "6/2/3", "8/8/8", "16/1/1", "12/2/4"])
@pytest.mark.parametrize("new", [[5, 5, 6], [16, 17, 1], [10, 11, 22], [33, 31, 64], [60, 65, 4], [1, 128, 130], [255, 1, 300]])
@pytest.mark.parametrize("prefix", [20, 150])
def test_rows_around_what_is_few(api, heads, new, prefix):
    step = Step(api, [prefix + 7 * i for i in range(3)] + [40], new + [18], *HEADS[heads], 64, 128, page=32, seed=sum(new), pad=2)
    run(api, hide(step, [0, 3], [prefix]), [0, 3], [prefix])


# one long prefix that many blocks have a part of; chunks whose own parts are long and cut too; both among others
LONG = {"64 single rows behind 16k": ([16000 + 37 * i for i in range(64)], [1] * 64, [0, 64], [16000]),
        "300 rows behind 4k": ([4100 + i for i in range(300)], [1, 1, 1, 0, 2] * 60, [0, 300], [4100]),
        "chunks behind 16k": ([16001, 16001 + 900, 17500, 16100, 16300, 16001, 18200, 16444], [40, 66, 80, 47, 51, 73, 1, 60],
                              [0, 8], [16001]),
        "chunks behind 8k, others": ([50, 8192 + 3000, 8192, 8192 + 1500, 3000, 2000, 2100, 900], [300, 150, 40, 77, 64, 1, 200, 5],
                                     [1, 4, 4, 7], [8192, 0, 2000])}


@pytest.mark.parametrize("name", LONG)
@pytest.mark.parametrize("heads,dims", [("8/4/2", (128, 128)), ("16/2/4", (64, 128)), ("16/1/1", (64, 64))])
def test_long_prefixes_and_own_parts(api, name, heads, dims):
    past, new, groups, prefix = LONG[name]
    step = Step(api, past, new, *HEADS[heads], *dims, page=64, seed=len(name), pad=2)
    run(api, hide(step, groups, prefix), groups, prefix)


@pytest.mark.parametrize("name", ["64 single rows behind 16k", "chunks behind 16k"])
def test_long_prefixes_with_any_workspace(api, name):
    past, new, groups, prefix = LONG[name]
    step = hide(Step(api, past, new, 8, 4, 2, 64, 64, page=128, seed=2, pad=1), groups, prefix)
    first, lse = run(api, step, groups, prefix)
    nbytes = api.diffqkv_extend_shared_workspace_bytes(api.make_shape(len(past), 8, 4, 2, 64, 64, BF16, BF16, 1.0), step.total_q)
    for fill in (0, 255):
        ws = torch.full((nbytes,), fill, dtype=torch.uint8, device="cuda")
        again, lse2 = run(api, step, groups, prefix, workspace=ws)
        assert torch.equal(first, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("k_std", [10.0, 40.0])
@pytest.mark.parametrize("past,new,prefix", [([900, 940, 905], [3, 140, 1], 890), ([900, 940, 905], [3, 1, 1], 890),
                                             ([9000, 9940, 9005], [60, 140, 71], 8990)])
def test_peaked_scores(api, k_std, past, new, prefix):
    """One of the two parts, and one of a cut one's, has nearly all of the weight."""
    step = Step(api, past, new, 8, 2, 4, 128, 128, seed=4, k_std=k_std)
    run(api, hide(step, [0, 3], [prefix]), [0, 3], [prefix])


@pytest.mark.parametrize("prefix,own,new", [(256, 50, 1), (256, 50, 90), (9000, 40, 1), (9000, 2000, 90)])
@pytest.mark.parametrize("where", ["prefix", "own", "both", "start"])
def test_parts_of_minus_infinity(api, prefix, own, new, where):
    """Keys of -inf (queries above 0): a part, or parts of a cut one, from which nothing comes."""
    step = Step(api, [prefix + own, prefix + own + 10], [new, new], 4, 2, 2, 64, 64, seed=2)
    step.q[:] = step.q.abs() + 0.1
    gone = {"prefix": slice(0, prefix), "own": slice(prefix, None), "both": slice(0, None), "start": slice(0, prefix - 100)}[where]
    for b in range(2):
        step.k_tok[b][gone] = -math.inf
    hide(step, [0, 2], [prefix])
    out, lse = torch.empty((2 * new, 4, 64), dtype=F32, device="cuda"), torch.empty((2 * new, 4), dtype=F32, device="cuda")
    api.diffqkv_extend_shared(step.q, step.cu, step.cache, ints([0, 2]), ints([prefix]), 2, 2, 0.125, out=out, lse=lse)
    if where == "both":
        assert bool((out == 0).all()) and bool((lse == -math.inf).all())
        return
    for b in range(2):  # bounds as in ranged.check
        past, t = step.past[b], step.total[b]
        sees = visible(past, new, t)
        sees[:, gone] = False
        ref, ref_lse, mean_abs, big = attend64(step.q[b * new:(b + 1) * new], step.k_tok[b], step.v_tok[b], 0.125, sees)
        score = (64 + 16) * 2.0 ** -24 * max(big, 1.0)
        weight = 2 * score + (t + 16) * 2.0 ** -24 + HALF_STEP[BF16]
        weight = (weight + 2.0 ** -21 + 2.0 ** -22 * ref_lse.abs() * 1.4427)[..., None]
        bound = weight * mean_abs * (1 + weight)
        bound = bound + HALF_STEP[F32] * (ref.abs() + bound)
        assert bool(((out[b * new:(b + 1) * new].double() - ref).abs() <= bound).all())
        bound = score + (t + 16) * 2.0 ** -24 + 2.0 ** -21 * ref_lse.abs() + 2.0 ** -21
        assert bool(((lse[b * new:(b + 1) * new].double() - ref_lse).abs() <= bound).all())


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


@pytest.mark.parametrize("long", [False, True])
def test_sequences_that_do_not_fit(api, long):
    """Reported and skipped; the others are as they would be, those behind a prefix of misfits too."""
    far, rows = (9000, [60, 40, 75, 90, 55]) if long else (0, [3, 40, 1, 1, 20])

    def call(groups, prefix, lens=None, bad=()):
        step = Step(api, [far + 300, far + 310, far + 290, 50, 40], rows, 8, 2, 4, 128, 128, seed=7, pad=1)
        share(step, [0, 3, 5], [far + 200, 40])
        if lens:
            step.lens.copy_(ints(lens))
        out, status = torch.full((step.total_q, 8, 128), 77.0, dtype=BF16, device="cuda"), ints([0])
        api.diffqkv_extend_shared(step.q, step.cu, step.cache, ints(groups), ints(prefix), 2, 4, 0.1, out=out, dev_status=status)
        assert int(status.item()) == (1 << api.ERR_INDEX if bad else 0)
        for b in bad:
            assert bool((out[step.cu_host[b]:step.cu_host[b + 1]] == 77.0).all()), b
        assert bool((out[step.rows:] == 77.0).all())
        check(step, out, None, 0.1, joined=True, only=[b for b in range(5) if b not in bad])

    call([0, 3], [far + 200])
    call([0, 3], [far + 200], lens=[far + 300, -1, far + 290, 50, 40], bad=[1])   # a denied sequence
    call([0, 3], [far + 200], lens=[far + 300, far + 199, far + 290, 50, 40], bad=[1])
    call([0, 3], [far + 200], lens=[far + 199, far + 310, far + 290, 50, 40], bad=[0])  # the one that would lend the prefix
    call([0, 3, 5], [far + 200, 40])
    call([0, 3, 5], [far + 200, 45], bad=[4])                                     # a prefix longer than the cache of one
    call([0, 3, 5], [far + 200, -1], bad=[3, 4])
    call([0, 3, 9], [far + 200, 0], bad=[3, 4])                                   # a group that ends outside of the batch
    call([-1, 3], [far + 200], bad=[0, 1, 2])
    call([0, 3, 5], [far + 200, 1 << 30], bad=[3, 4])


@pytest.mark.parametrize("bad", [None, 1, 2])
def test_a_few_rows_in_all(api, bad):
    """Steps that one kernel takes alone, with a sequence that does not fit among them."""
    step = Step(api, [300, 310, 290, 50], [1, 2, 2, 1], 8, 2, 4, 128, 128, seed=7, pad=2)
    hide(step, [0, 3], [200])
    if bad is not None:
        step.lens[bad] = -1 if bad == 2 else 199
    out, status = torch.full((step.total_q, 8, 128), 77.0, dtype=BF16, device="cuda"), ints([0])
    api.diffqkv_extend_shared(step.q, step.cu, step.cache, ints([0, 3]), ints([200]), 2, 4, 0.1, out=out, dev_status=status)
    assert int(status.item()) == (0 if bad is None else 1 << api.ERR_INDEX)
    check(step, out, None, 0.1, joined=True, only=[b for b in range(4) if b != bad])
    if bad is not None:
        assert bool((out[step.cu_host[bad]:step.cu_host[bad + 1]] == 77.0).all())
    assert bool((out[step.rows:] == 77.0).all())


@pytest.mark.parametrize("heads", [(256, 1, 2), (132, 1, 4)])
def test_head_groups_too_wide_for_few_rows(api, heads):
    step = Step(api, [300, 290, 400], [1, 2, 3], *heads, 64, 128, seed=9, pad=2)
    run(api, hide(step, [0, 3], [280]), [0, 3], [280])


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
    run(api, hide(step, ends, prefix), ends, prefix)


def test_two_calls_at_once_and_other_streams(api):
    steps = [hide(Step(api, [5000 + i, 5050], [1 + i, 80], 16, 2, 4, 128, 128, seed=i), [0, 2], [4999]) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in steps]
    outs = [torch.zeros((s.total_q, 16, 128), dtype=BF16, device="cuda") for s in steps]
    cu, lens = ints([0, 2]), ints([4999])
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
                ([0, 5, 10, 0], [3, 1, 1, 40], [1, 1, 1], [0, 0]), ([600, 610, 650, 640], [30, 30, 30, 30], [0, 4, 4], [599, 0])]
    q = torch.zeros((cap, 8, 64), dtype=BF16, device="cuda")
    out = torch.full((cap, 8, 64), 77.0, dtype=BF16, device="cuda")
    steps = [hide(Step(api, p, n, 8, 2, 4, 64, 64, seed=3, room=60), g, l) for p, n, g, l in variants]
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
    for i in (0, 1, 2, 3, 0):
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


@pytest.mark.parametrize("seed", range(40))
def test_random_steps(api, seed):
    r = random.Random(seed)
    n_q, n_k, n_v = HEADS[r.choice(list(HEADS))]
    dims = r.choice([(128, 128), (64, 64), (64, 128)])
    n = r.randint(1, 12)
    ends = sorted(r.randint(0, n) for _ in range(r.randint(2, 5)))
    prefix = [r.choice([0, r.randint(1, 300), r.randint(1, 6000)]) for _ in ends[1:]]
    past = [r.randint(0, 300) for _ in range(n)]
    for g, p in enumerate(prefix):
        for b in range(ends[g], ends[g + 1]):
            past[b] = p + r.choice([0, r.randint(0, 200)])
    new = [r.choice([0, 1, 1, r.randint(1, 12), r.randint(1, 150), r.randint(1, 400)]) for _ in range(n)]
    step = Step(api, past, new, n_q, n_k, n_v, *dims, page=r.choice([8, 16, 32, 64, 128, 256]),
                layout=r.choice(["paged", "paged", "token", "flat"]), pad=r.randint(0, 3), seed=seed, room=r.randint(0, 50))
    run(api, hide(step, ends, prefix), ends, prefix)


def test_the_hook(api):
    """Which prefixes are read once shows in whose copy matters."""
    step = hide(Step(api, [600, 610], [2, 3], 8, 2, 4, 64, 64, seed=1), [0, 2], [590])
    out = torch.empty((5, 8, 64), dtype=BF16, device="cuda")
    cu, lens, status = ints([0, 2]), ints([590]), ints([0])
    for choice, shared in ((0, True), (1, True), (2, False)):
        api.extend_sharing(choice)
        status.zero_()
        api.diffqkv_extend_shared(step.q, step.cu, step.cache, cu, lens, 2, 4, 0.1, out=out, dev_status=status)
        assert (int(status.item()) == 0) == shared
        assert bool(torch.isfinite(out[:2]).all()) and bool(torch.isfinite(out).all()) == shared


def lends(api, past, new, prefix, heads="16/2/4", dims=(128, 128), slots=0):
    """Whether a group's prefix is read once by itself: the first sequence, without rows, has NaN in its place, the others have
    their own.  slots: sequences without rows behind it."""
    api.extend_sharing(0)
    step = Step(api, [prefix] + [prefix] * slots + past, [0] * (slots + 1) + new, *HEADS[heads], *dims, seed=prefix, pad=1)
    groups = [0, slots + 1 + len(past)]
    share(step, groups, [prefix], same_pages=False)
    blk, slot = step.place(0, 0, prefix)
    step.k[blk, :, slot] = math.nan
    out = torch.full((step.total_q, step.n_q, step.d_v), 77.0, dtype=BF16, device="cuda")
    api.diffqkv_extend_shared(step.q, step.cu, step.cache, ints(groups), ints([prefix]), step.n_k, step.n_v, 0.1, out=out)
    gone = torch.isnan(out[:step.rows])
    assert bool(gone.all()) or not bool(gone.any())
    if not bool(gone.any()):
        check(step, out, None, 0.1, joined=True)
    return bool(gone.all())


@pytest.mark.parametrize("new", [1, 2, 9, 100, 200])
@pytest.mark.parametrize("slots", [0, 1, 63])
def test_one_sequence_with_rows_reads_its_own(api, new, slots):
    assert not lends(api, [8200], [new], 8192, slots=slots)


@pytest.mark.parametrize("past,new", [(8192, 200), (8200, 480), (5000, 1), (5000, 17)])
def test_a_group_of_one_is_none(api, past, new):
    step = Step(api, [past, 70], [new, 3], 32, 4, 8, 128, 128, seed=new).fill()
    out = [torch.empty((step.total_q, 32, 128), dtype=F32, device="cuda") for _ in range(3)]
    for choice in range(3):
        api.extend_sharing(choice)
        api.diffqkv_extend_shared(step.q, step.cu, step.cache, ints([0, 1]), ints([5000]), 4, 8, 0.1, out=out[choice])
    assert torch.equal(out[0], out[2]) and not torch.equal(out[0], out[1])


@pytest.mark.parametrize("readers,prefix,shared", [(2, 511, False), (2, 512, True), (3, 255, False), (3, 256, True), (9, 63, False),
                                                   (9, 64, True), (70, 7, False), (70, 8, True)])
@pytest.mark.parametrize("slots", [0, 40, 200])
def test_few_rows_share_by_their_sequences(api, readers, prefix, shared, slots):
    """Sequences without rows do not count: among the first ones, that is; behind them as many as have rows at most."""
    assert lends(api, [prefix + i for i in range(readers)], [1] * readers, prefix, slots=slots) == shared


@pytest.mark.parametrize("readers,prefix,shared", [(2, 5398, False), (2, 5399, True), (5, 3758, False), (5, 3759, True), (2, 1024, False)])
@pytest.mark.parametrize("slots", [0, 20])
def test_long_chunks_share_by_their_sequences(api, readers, prefix, shared, slots):
    """(prefix - 1024) 32 (readers - 1) >= 700 rows, in chunks of a hundred rows of four heads."""
    assert lends(api, [prefix + i for i in range(readers)], [100] * readers, prefix, slots=slots) == shared
