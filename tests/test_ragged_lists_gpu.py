"""Ragged steps whose lengths or row lists do not fit: what is reported, what is written and, bit for bit, what is not."""
import math

import pytest
import torch

from ragged import BF16, F32, Step, attend64, check_extend, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2501_13629_b200 import api as _api
    return _api


CAP, ROW, PAGE, TOTAL = 64, 9, 8, 44  # tokens a sequence may have; the table's rows have a page more than that, and a
                                      # sequence of their own follows: what is written too far lands in memory of the test
LISTS = {
    # cu_q, past, and the sequences that fit and share no row with another that does
    "an early end far ahead": ([0, 40, 3, 8, 44], [10, 20, 50, 1], []),
    "an early end beyond the rows": ([0, 100, 3, 8, 44], [10, 20, 56, 1], [2, 3]),
    "an end before the beginning": ([0, 20, 19, 30, 44], [10, 20, 40, 50], [3]),
    "the last beyond the rows": ([0, 20, 24, 30, 45], [10, 20, 58, 1], [0, 1, 2]),
    "a negative beginning": ([-3, 20, 24, 30, 44], [10, 20, 58, 1], [1, 2, 3]),
    "a negative end": ([0, -3, 20, 30, 44], [10, 20, 54, 1], [2, 3]),
    "the largest and smallest numbers": ([0, 2 ** 31 - 1, -2 ** 31, 4, 8], [10, 20, 30, 60], [3]),
    "too long by one": ([0, 10, 20, 30, 44], [55, 54, 10, 51], [1, 2]),
    "lengths out of range": ([0, 10, 20, 30, 44], [2 ** 31 - 1, -1, 54, -2 ** 31], [2]),
}


def claims(cu, past):
    """Rows and positions of every sequence that fits, by the header's rule."""
    fit = {}
    for b, p in enumerate(past):
        lo, hi = cu[b], cu[b + 1]
        if 0 <= lo <= hi <= TOTAL and p >= 0 and p + hi - lo <= CAP:
            fit[b] = (lo, hi, p)
    return fit


def pools(n_k, n_v, d_qk, d_v, dtype, paged, seed):
    """Four sequences and one that the step does not have, all positions filled."""
    g = torch.Generator("cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    if not paged:  # contiguous, each with room behind its capacity
        return rand(5, n_k, CAP + 24, d_qk), rand(5, n_v, CAP + 24, d_v), None
    table = torch.randperm(5 * ROW, generator=g, device="cuda").to(torch.int32).view(5, ROW)
    return rand(5 * ROW, n_k, PAGE, d_qk), rand(5 * ROW, n_v, PAGE, d_v), table


def cache_of(api, k, v, table, past):
    if table is None:
        return api.KVCache(k[:, :, :CAP], v[:, :, :CAP], ints(past), CAP)
    return api.KVCache(k, v, ints(past), CAP, page_table=table[:4], page_size=PAGE)


def place(table, b, start, stop):
    t = torch.arange(start, stop, device="cuda")
    if table is None:
        return torch.full_like(t, b), t
    return table[b].long()[t // PAGE], t % PAGE


def bits(x):
    return x.contiguous().view(torch.uint8)


def test_the_lists_are_what_they_say():
    for cu, past, alone in LISTS.values():
        fit = claims(cu, past)
        assert len(fit) < 4 and set(alone) <= set(fit)
        for b in alone:
            lo, hi, _ = fit[b]
            assert hi > lo and all(c == b or z <= lo or hi <= a for c, (a, z, _) in fit.items())


@pytest.mark.parametrize("name", LISTS)
@pytest.mark.parametrize("paged", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rope_append(api, name, paged, dtype):
    cu, past, alone = LISTS[name]
    n_q, n_k, n_v, d = 4, 2, 2, 64
    k, v, table = pools(n_k, n_v, d, d, dtype, paged, 1)
    g = torch.Generator("cuda").manual_seed(2)
    q, k_new, v_new = (torch.randn((TOTAL, h, d), generator=g, device="cuda").to(dtype) for h in (n_q, n_k, n_v))
    out = torch.full((TOTAL, n_q, d), 5.0, dtype=dtype, device="cuda")
    want_k, want_v, want_q = k.clone(), v.clone(), out.clone()
    status = ints([0])
    api.diffqkv_rope_append(q, k_new, v_new, ints(cu), cache_of(api, k, v, table, past), None, q_out=out, dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 1 << api.ERR_INDEX
    fit = claims(cu, past)
    for b, (lo, hi, p) in fit.items():
        blk, slot = place(table, b, p, p + hi - lo)
        if b in alone:
            want_k[blk, :, slot], want_v[blk, :, slot], want_q[lo:hi] = k_new[lo:hi], v_new[lo:hi], q[lo:hi]
        else:  # a row of several: its places may be written
            want_k[blk, :, slot], want_v[blk, :, slot], want_q[lo:hi] = k[blk, :, slot], v[blk, :, slot], out[lo:hi]
            turned = (out[lo:hi] == q[lo:hi]).flatten(1).all(1)
            assert bool((turned | (out[lo:hi] == 5.0).flatten(1).all(1)).all())
    assert torch.equal(bits(k), bits(want_k)) and torch.equal(bits(v), bits(want_v)) and torch.equal(bits(out), bits(want_q))


@pytest.mark.parametrize("name", LISTS)
@pytest.mark.parametrize("choice,dtype,d_qk", [(0, BF16, 128), (0, F32, 64), (2, BF16, 64), (1, F32, 64), (0, BF16, 96)])
def test_extend(api, name, choice, dtype, d_qk):
    """Tensor cores, tiles on FMAs, a block a row."""
    cu, past, alone = LISTS[name]
    n_q, n_k, n_v, d_v = 8, 2, 4, 128
    k, v, table = pools(n_k, n_v, d_qk, d_v, dtype, True, 3)
    q = torch.randn((TOTAL, n_q, d_qk), generator=torch.Generator("cuda").manual_seed(4), device="cuda").to(dtype)
    out = torch.full((TOTAL, n_q, d_v), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((TOTAL, n_q), 7.0, dtype=F32, device="cuda")
    status = ints([0])
    api.extend_kernel(choice)
    try:
        api.diffqkv_extend(q, ints(cu), cache_of(api, k, v, table, past), n_k, n_v, 0.125, out=out, lse=lse,
                           dev_status=status)
    finally:
        api.extend_kernel(0)
    torch.cuda.synchronize()
    assert int(status.item()) == 1 << api.ERR_INDEX
    fit = claims(cu, past)
    free = torch.ones(TOTAL, dtype=torch.bool, device="cuda")
    for lo, hi, _ in fit.values():
        free[lo:hi] = False
    assert bool((out[free] == 7.0).all()) and bool((lse[free] == 7.0).all())
    for b in alone:
        lo, hi, p = fit[b]
        blk, slot = place(table, b, 0, p + hi - lo)
        s = Step.__new__(Step)
        s.past, s.new, s.total, s.cu_host, s.q, s.d_qk, s.dtype = [p], [hi - lo], [p + hi - lo], [0], q[lo:hi], d_qk, dtype
        s.k_tok, s.v_tok = [k[blk, :, slot]], [v[blk, :, slot]]
        check_extend(s, out[lo:hi], lse[lo:hi], 0.125)


def test_joined_splits(api):
    """Splits along the tokens: a row whose sequence the others' ends do not lead to."""
    step = Step(api, [0, 5, 900], [0, 0, 20], 8, 2, 4, 64, 64, dtype=F32, seed=5, pad=3).fill()
    q = torch.cat([step.q[20:], step.q[:20]])  # rows 3 .. 22
    out, status = torch.full((23, 8, 64), 7.0, dtype=F32, device="cuda"), ints([0])
    lse = torch.full((23, 8), 7.0, dtype=F32, device="cuda")
    before = api.launch_count()
    api.diffqkv_extend(q, ints([0, 100, 3, 23]), step.cache, 2, 4, 0.125, out=out, lse=lse, dev_status=status)
    torch.cuda.synchronize()
    assert api.launch_count() - before == 2 and api.last_extend_kernel() == 2
    assert int(status.item()) == 1 << api.ERR_INDEX
    assert bool((out[:3] == 7.0).all()) and bool((lse[:3] == 7.0).all())
    check_extend(step, out[3:], lse[3:], 0.125)


@pytest.mark.parametrize("choice,dtype,d_qk", [(0, BF16, 64), (0, F32, 64), (1, F32, 64)])
def test_the_last_of_many_sequences_is_reported(api, choice, dtype, d_qk):
    step = Step(api, [3] * 600, [1] * 600, 4, 2, 2, d_qk, 64, dtype=dtype, seed=6).fill()
    step.lens[599] = step.max_seqlen
    out, status = torch.full((600, 4, 64), 7.0, dtype=dtype, device="cuda"), ints([0])
    api.extend_kernel(choice)
    try:
        api.diffqkv_extend(step.q, step.cu, step.cache, 2, 2, 0.125, out=out, dev_status=status)
    finally:
        api.extend_kernel(0)
    torch.cuda.synchronize()
    assert int(status.item()) == 1 << api.ERR_INDEX
    assert bool((out[599] == 7.0).all())
    step.new[599] = 0
    check_extend(step, out, None, 0.125)


@pytest.mark.parametrize("src,dst", [(-1, -1), (-1, 2), (1, -1), (-2 ** 31, -2 ** 31), (6, 6)])
def test_a_copy_without_pages_is_reported(api, src, dst):
    k, v = (torch.randn((6, 2, 16, 64), device="cuda").to(BF16) for _ in range(2))
    cache = api.KVCache(k, v, ints([0]), 16, page_table=ints([[0]]), page_size=16)
    want_k, want_v, status = k.clone(), v.clone(), ints([0])
    want_k[5], want_v[5] = k[4], v[4]
    api.diffqkv_pages_copy(ints([src, 4]), ints([dst, 5]), cache, 2, 2, dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 1 << api.ERR_INDEX
    assert torch.equal(k, want_k) and torch.equal(v, want_v)


@pytest.mark.parametrize("cu,past,fits", [
    ([0, 10, 20, 30, 44], [55, 54, 10, 51], [0, 1, 1, 0]),                  # past + n up to the capacity, and one more
    ([0, 10, 20, 30, 44], [2 ** 31 - 1, -1, 54, -2 ** 31], [0, 0, 1, 0]),
    ([-3, 20, 24, 30, 44], [10, 20, 58, 1], [0, 1, 1, 1]),
    ([0, 20, 19, 30, 30], [10, 20, 40, 50], [1, 0, 1, 1]),
    ([0, 0, 0, 0, 1], [-1, 65, 64, 64], [1, 1, 1, 0]),                      # nothing to write fits anywhere
])
def test_reserve_grants_what_the_other_calls_write(api, cu, past, fits):
    """A table row has room for 72 tokens, a sequence for 64."""
    k, v, _ = pools(2, 2, 64, 64, BF16, True, 7)
    table, refs = torch.full((4, ROW), -1, dtype=torch.int32, device="cuda"), torch.zeros(5 * ROW, dtype=torch.int32, device="cuda")
    granted, status = ints([9] * 4), ints([0])
    cache = api.KVCache(k, v, ints(past), CAP, page_table=table, page_size=PAGE)
    api.diffqkv_pages_reserve(ints(cu), cache, refs, 2, 2, granted=granted, dev_status=status)
    torch.cuda.synchronize()
    assert granted.tolist() == fits
    assert int(status.item()) == 1 << api.ERR_INDEX
    want, used = [[-1] * ROW for _ in range(4)], 0
    for b, ok in enumerate(fits):
        lo, hi = cu[b], cu[b + 1]
        if ok and hi > lo:
            for e in range(past[b] // PAGE, -(-(past[b] + hi - lo) // PAGE)):
                want[b][e], used = used, used + 1
    assert table.tolist() == want
    assert refs.tolist() == [1] * used + [0] * (5 * ROW - used)


def test_denied_sequences_are_left_out_of_a_captured_step(api):
    """reserve -> lengths of the granted ones -> rope_append -> extend, captured.  Sequence 1 shares a half-filled page with
    sequence 0 and gets no page of its own once the pool has run out: sequence 0's tokens stay what they were."""
    n_q, n_k, n_v, d, page, n_pages = 4, 2, 2, 64, 16, 4
    g = torch.Generator("cuda").manual_seed(8)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(BF16)  # noqa: E731
    k, v = rand(n_pages, n_k, page, d), rand(n_pages, n_v, page, d)
    table, refs, lens = ints([[0, -1], [0, -1], [1, -1]]), ints([2, 1, 0, 0]), ints([5, 5, 9])
    cu, granted, status, seen = ints([0, 1, 2, 3]), ints([0] * 3), ints([0]), ints([0] * 3)
    q, k_new, v_new = rand(3, n_q, d), rand(3, n_k, d), rand(3, n_v, d)
    out = torch.zeros((3, n_q, d), dtype=BF16, device="cuda")
    cache = api.KVCache(k, v, lens, 2 * page, page_table=table, page_size=page)
    writes = api.KVCache(k, v, seen, 2 * page, page_table=table, page_size=page)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")

    def step():
        api.diffqkv_pages_reserve(cu, cache, refs, n_k, n_v, granted=granted, workspace=ws, dev_status=status)
        seen.copy_(torch.where(granted > 0, lens, -1))
        api.diffqkv_rope_append(q, k_new, v_new, cu, writes, None, q_out=q, dev_status=status)
        api.diffqkv_extend(q, cu, writes, n_k, n_v, 0.125, out=out, workspace=ws, dev_status=status)

    state = [x.clone() for x in (k, v, table, refs, lens)]
    step()  # two free pages: 0 and 1 write, each gets a copy
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and granted.tolist() == [1, 1, 1] and table.tolist() == [[2, -1], [3, -1], [1, -1]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for x, y in zip((k, v, table, refs, lens), state):
        x.copy_(y)
    refs.copy_(ints([2, 1, 1, 0]))  # one free page
    status.zero_(), out.fill_(3.0)
    graph.replay()
    torch.cuda.synchronize()
    assert granted.tolist() == [1, 0, 1] and int(status.item()) == (1 << api.ERR_PAGES) | (1 << api.ERR_INDEX)
    assert table.tolist() == [[3, -1], [0, -1], [1, -1]] and refs.tolist() == [1, 1, 1, 1]
    want_k, want_v = state[0].clone(), state[1].clone()
    for pool, new in ((want_k, k_new), (want_v, v_new)):
        pool[3] = pool[0]  # sequence 0's copy
        pool[3, :, 5], pool[1, :, 9] = new[0], new[2]
    assert torch.equal(k, want_k) and torch.equal(v, want_v)
    assert bool((out[1] == 3.0).all())
    for b, (blk, n) in ((0, (3, 6)), (2, (1, 10))):
        ref, _, _, _ = attend64(q[b:b + 1], k[blk, :, :n].transpose(0, 1), v[blk, :, :n].transpose(0, 1), 0.125, n - 1)
        # a weight is off by half a step of bf16 and little besides, the result by another
        assert bool(((out[b:b + 1].double() - ref).abs() <= 3 * 2.0 ** -8 * v[blk, :, :n].double().abs().amax()).all())


def test_rope_append_of_many_sequences_one_out_of_order(api):
    """More sequences than a block has threads; one end far ahead moves the count of ends for every row before it."""
    n = 600
    k, v = (torch.zeros((n, 2, 4, 64), dtype=BF16, device="cuda") for _ in range(2))
    cu = list(range(n + 1))
    cu[301] = 590  # sequence 300 gets 290 rows and does not fit, 301 ends before it begins, the others have their row
    lens = [i % 4 for i in range(n)]
    lens[599] = 4  # full
    g = torch.Generator("cuda").manual_seed(9)
    q, k_new, v_new = (torch.randn((n, h, 64), generator=g, device="cuda").to(BF16) for h in (4, 2, 2))
    out, status = torch.full((n, 4, 64), 5.0, dtype=BF16, device="cuda"), ints([0])
    api.diffqkv_rope_append(q, k_new, v_new, ints(cu), api.KVCache(k, v, ints(lens), 4), None, q_out=out, dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 1 << api.ERR_INDEX
    want_k, want_v, want_q = torch.zeros_like(k), torch.zeros_like(v), torch.full_like(out, 5.0)
    for b in range(n):
        if b not in (300, 301, 599):
            want_k[b, :, lens[b]], want_v[b, :, lens[b]], want_q[b] = k_new[b], v_new[b], q[b]
    assert torch.equal(k, want_k) and torch.equal(v, want_v) and torch.equal(out, want_q)
