"""The ragged-batch calls where element offsets pass 2^31, through each of the strides: blocks, tokens and heads."""
import pytest
import torch

from ragged import BF16, F32, Step, check_extend, ints

pytestmark = pytest.mark.gpu

FAR = 1 << 31


@pytest.fixture(scope="module")
def api():
    from paper_2501_13629_b200 import api as _api
    return _api


def pools(kind, n_k, n_v, d):
    """(K, V, table, page, max_seqlen, past): the last tokens of the sequence lie behind FAR elements in both pools."""
    if kind == "blocks":
        pages, page = FAR // (min(n_k, n_v) * 128 * d) + 3, 128
        k, v = (torch.zeros((pages, h, page, d), dtype=BF16, device="cuda") for h in (n_k, n_v))
        assert all((pages - 1) * x.stride(0) > FAR for x in (k, v))
        return k, v, ints([[0, pages - 1]]), page, 256, 200
    if kind == "tokens":  # a narrow part of wide rows, no pages
        wide = 8192
        tokens = FAR // wide + 40
        k, v = (torch.zeros((1, tokens, wide), dtype=BF16, device="cuda")[:, :, :h * d].unflatten(2, (h, d)).transpose(1, 2)
                for h in (n_k, n_v))
        assert all((tokens - 30) * x.stride(2) > FAR for x in (k, v))
        return k, v, None, 0, tokens, tokens - 20
    per = FAR // (min(n_k, n_v) - 1) // (32 * d) + 2  # heads outermost: the last one begins behind FAR
    k, v = (torch.zeros((h, per, 32, d), dtype=BF16, device="cuda").transpose(0, 1) for h in (n_k, n_v))
    assert all((h - 1) * x.stride(1) > FAR for h, x in ((n_k, k), (n_v, v)))
    return k, v, ints([[5, per - 1, 0, 7]]), 32, 128, 40


@pytest.mark.parametrize("kind", ["blocks", "tokens", "heads"])
@pytest.mark.parametrize("choice", [0, 1, 2])
@pytest.mark.parametrize("new", [3, 70])
def test_rope_append_and_extend(api, kind, choice, new):
    n_q, n_k, n_v, d = 8, 2, 4, 128
    if kind == "tokens":
        new = min(new, 20)
    k, v, table, page, max_seqlen, past = pools(kind, n_k, n_v, d)
    new = min(new, max_seqlen - past)
    g = torch.Generator("cuda").manual_seed(1)
    s = Step.__new__(Step)
    s.past, s.new, s.total, s.cu_host, s.d_qk, s.dtype = [past], [new], [past + new], [0, new], d, BF16
    rand = lambda *x: torch.randn(x, generator=g, device="cuda").to(BF16)  # noqa: E731
    s.q, s.k_tok, s.v_tok = rand(new, n_q, d), [rand(past + new, n_k, d)], [rand(past + new, n_v, d)]
    t = torch.arange(past + new, device="cuda")
    blk, slot = (torch.zeros_like(t), t) if table is None else (table[0].long()[t // page], t % page)
    k[blk[:past], :, slot[:past]], v[blk[:past], :, slot[:past]] = s.k_tok[0][:past], s.v_tok[0][:past]
    cache = api.KVCache(k, v, ints([past]), max_seqlen, page_table=table, page_size=page)
    cu, status = ints([0, new]), ints([0])
    q = api.diffqkv_rope_append(s.q, s.k_tok[0][past:], s.v_tok[0][past:], cu, cache, None, dev_status=status)
    assert torch.equal(q, s.q)
    assert torch.equal(k[blk[past:], :, slot[past:]], s.k_tok[0][past:])
    assert torch.equal(v[blk[past:], :, slot[past:]], s.v_tok[0][past:])
    out, lse = torch.empty((new, n_q, d), dtype=F32, device="cuda"), torch.empty((new, n_q), dtype=F32, device="cuda")
    api.extend_kernel(choice)
    try:
        api.diffqkv_extend(q, cu, cache, n_k, n_v, d ** -0.5, out=out, lse=lse, dev_status=status)
        assert api.last_extend_kernel() == (choice or 3)
    finally:
        api.extend_kernel(0)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    check_extend(s, out, lse, d ** -0.5)


@pytest.mark.parametrize("kind", ["blocks", "heads"])
def test_pages(api, kind):
    """Copy, copy on write and compaction from and to pages behind 2^31 elements."""
    n_k, n_v, d = 2, 4, 128
    k, v, _, page, _, _ = pools(kind, n_k, n_v, d)
    n = k.shape[0]
    last = n - 1
    k[3], v[3] = 1.5, 2.5
    k[last - 1], v[last - 1] = 3.5, 4.5
    table, refs, lens = ints([[last - 1, -1], [last - 1, -1]]), torch.ones(n, dtype=torch.int32, device="cuda"), ints([5, 5])
    refs[last - 1], refs[last] = 2, 0  # one page is free: the last
    cache, status = api.KVCache(k, v, lens, 2 * page, page_table=table, page_size=page), ints([0])
    same = lambda at, a, b: bool((k[at] == a).all()) and bool((v[at] == b).all())  # noqa: E731
    api.diffqkv_pages_copy(ints([3]), ints([last]), cache, n_k, n_v, dev_status=status)
    torch.cuda.synchronize()
    assert same(last, 1.5, 2.5) and same(3, 1.5, 2.5) and same(2, 0, 0) and same(4, 0, 0)
    api.diffqkv_pages_reserve(ints([0, 1, 1]), cache, refs, n_k, n_v, dev_status=status)
    torch.cuda.synchronize()
    assert table.tolist() == [[last, -1], [last - 1, -1]] and same(last, 3.5, 4.5) and same(last - 1, 3.5, 4.5)
    assert not bool(k[4:last - 1].any()) and not bool(v[4:last - 1].any())
    refs[0:2], refs[last - 1], refs[last] = 0, 1, 1  # the two holes in front take the last two
    live = ints([0])
    api.diffqkv_pages_compact(cache, refs, n_k, n_v, live=live, dev_status=status)
    torch.cuda.synchronize()
    assert int(live.item()) == n - 2 and table.tolist() == [[1, -1], [0, -1]]
    assert same(0, 3.5, 4.5) and same(1, 3.5, 4.5) and same(2, 0, 0) and int(status.item()) == 0


@pytest.mark.parametrize("n,choice", [(130, 0), (2, 0), (2, 2)])
def test_rows_behind_2_to_31_elements(api, n, choice):
    """Queries and results of more than 2^31 elements: sequences of n rows, the last ones checked."""
    n_q, n_k, n_v, d = 128, 8, 8, 128
    batch = FAR // (n_q * d * n) + 3
    if batch > 65535:
        batch, n = 65535, 3
    rows = batch * n
    assert rows * n_q * d > FAR
    g = torch.Generator("cuda").manual_seed(2)
    k, v = (torch.randn((1, h, 256, d), generator=g, device="cuda").to(BF16) for h in (n_k, n_v))
    table, cu = torch.zeros((batch, 1), dtype=torch.int32, device="cuda"), ints([i * n for i in range(batch + 1)])
    lens = torch.full((batch,), 60, dtype=torch.int32, device="cuda")
    cache, status = api.KVCache(k, v, lens, 256, page_table=table, page_size=256), ints([0])
    q = torch.zeros((rows, n_q, d), dtype=BF16, device="cuda")
    q[-2 * n:] = torch.randn((2 * n, n_q, d), generator=g, device="cuda").to(BF16)
    kept = q[-2 * n:].clone()
    k_new, v_new = torch.zeros((rows, n_k, d), dtype=BF16, device="cuda"), torch.zeros((rows, n_v, d), dtype=BF16, device="cuda")
    for i, x in ((0, k_new), (1, v_new)):  # all sequences share the page and write the same
        x.view(batch, n, 8, d)[:] = torch.randn((n, 8, d), generator=g, device="cuda").to(BF16)
    api.diffqkv_rope_append(q, k_new, v_new, cu, cache, None, q_out=q, dev_status=status)
    assert torch.equal(q[-2 * n:], kept)
    assert torch.equal(k[0, :, 60:60 + n].transpose(0, 1), k_new[-n:]) and torch.equal(v[0, :, 60:60 + n].transpose(0, 1), v_new[-n:])
    out = torch.zeros((rows, n_q, d), dtype=BF16, device="cuda")
    lse = torch.zeros((rows, n_q), dtype=F32, device="cuda")
    api.extend_kernel(choice)
    try:
        api.diffqkv_extend(q, cu, cache, n_k, n_v, d ** -0.5, out=out, lse=lse, dev_status=status)
    finally:
        api.extend_kernel(0)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    s = Step.__new__(Step)
    s.past, s.new, s.total, s.cu_host, s.q, s.d_qk, s.dtype = [60, 60], [n, n], [60 + n, 60 + n], [0, n], kept, d, BF16
    s.k_tok, s.v_tok = [k[0, :, :60 + n].transpose(0, 1)] * 2, [v[0, :, :60 + n].transpose(0, 1)] * 2
    check_extend(s, out[-2 * n:], lse[-2 * n:], d ** -0.5)
