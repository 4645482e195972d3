"""diffqkv_norm_rope_append: norms of query and key heads with the rotation and the cache write, against float64."""
import math

import pytest
import torch

from ragged import BF16, F32, HALF_STEP, Step, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2501_13629_b200 import api as _api
    return _api


def normed64(x, weight, eps, offset):
    y = x.double()
    y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps)
    if weight is not None:
        return y * (weight.double() + offset)
    return y * (offset if offset else 1.0)


def turned64(y, pos, inv_freq, interleaved, magnitude):
    """(the turned heads, what their channels are sums of)"""
    z, size = y.clone(), y.abs()
    if inv_freq is None:
        return z, size
    half = inv_freq.numel()
    angle = torch.outer(pos.double(), inv_freq)[:, None]
    i = torch.arange(half, device=y.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    u, v = y[..., a], y[..., b]
    z[..., a] = magnitude * (u * angle.cos() - v * angle.sin())
    z[..., b] = magnitude * (v * angle.cos() + u * angle.sin())
    size[..., a] = size[..., b] = (u.abs() + v.abs()) * magnitude
    return z, size


def check(out, x, weight, eps, offset, pos, inv, interleaved, magnitude, what):
    """In steps of 2^-23: the sum of d squares is off by (d + 1) / 2 of itself, its root by half of that; mean, eps, root
    (rsqrt is good to 2 steps), the factor, the weight and the two products by one each (8); cos and sin by 4 (see the
    rotation's own test), its products and difference by 2.  Then one rounding to the type."""
    d = x.shape[-1]
    y, size = turned64(normed64(x, weight, eps, offset), pos, inv, interleaved, magnitude)
    loss = ((d + 1) / 4 + 14) * 2.0 ** -23 * size
    bound = loss + HALF_STEP[out.dtype] * (y.abs() + loss) + 1e-38
    err = (out.double() - y).abs()
    assert bool((err <= bound).all()), f"{what}: {float((err / bound).max()):.2f} times the bound"


def run(api, step, rot, interleaved=False, magnitude=1.0, positions=None, in_place=False, fused=False, want_q=True,
        weights="shared", weight_dtype=None, eps=1e-6, offset=0.0, std=1.0, stream=None):
    s = step
    inv = None if rot == 0 else api.rope_frequencies(rot, 500000.0, device="cuda")[0]
    k_new = torch.full((s.total_q, s.n_k, s.d_qk), math.nan, dtype=s.dtype, device="cuda")
    v_new = torch.full((s.total_q, s.n_v, s.d_v), math.nan, dtype=s.dtype, device="cuda")
    for b, p in enumerate(s.past):
        k_new[s.cu_host[b]:s.cu_host[b + 1]] = (s.k_tok[b][p:].float() * std).to(s.dtype)
        v_new[s.cu_host[b]:s.cu_host[b + 1]] = s.v_tok[b][p:]
    q = (s.q.float() * std).to(s.dtype)
    gen = torch.Generator("cuda").manual_seed(rot + s.d_qk)
    wt = weight_dtype or s.dtype
    make = lambda *n: (torch.randn(n, generator=gen, device="cuda") * 0.3 + 1 - offset).to(wt)  # noqa: E731
    if weights == "shared":
        qw, kw = make(s.d_qk), make(s.d_qk)
    elif weights == "heads":
        qw, kw = make(s.n_q, s.d_qk), make(s.n_k, s.d_qk)
    elif weights == "sliced":  # a wider table's columns
        qw, kw = make(s.n_q, 2 * s.d_qk)[:, s.d_qk:], make(s.n_k, 3 * s.d_qk)[:, :s.d_qk]
    elif weights == "keys":
        qw, kw = None, make(s.d_qk)
    else:
        qw = kw = None
    if fused:  # slices of one projection's output
        both = torch.cat([x.reshape(s.total_q, -1) for x in (q, k_new, v_new)], 1)
        cut = [s.n_q * s.d_qk, (s.n_q + s.n_k) * s.d_qk]
        q = both[:, :cut[0]].unflatten(1, (s.n_q, s.d_qk))
        k_new = both[:, cut[0]:cut[1]].unflatten(1, (s.n_k, s.d_qk))
        v_new = both[:, cut[1]:].unflatten(1, (s.n_v, s.d_v))
    out = q if in_place else torch.full((s.total_q, s.n_q, s.d_qk), 5.0, dtype=s.dtype, device="cuda")
    want_k, want_v, q0 = s.k.clone(), s.v.clone(), q.clone()
    status = ints([0])
    torch.cuda.synchronize()
    got = api.diffqkv_norm_rope_append(q if want_q else None, k_new, v_new, s.cu, s.cache, inv, qw if want_q else None, kw, eps,
                                       weight_offset=offset, interleaved=interleaved, magnitude=magnitude,
                                       positions=positions, q_out=out if want_q else None, dev_status=status, stream=stream)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and (got is out if want_q else got is None)
    for b, (p, n) in enumerate(zip(s.past, s.new)):
        lo, hi = s.cu_host[b], s.cu_host[b + 1]
        if n == 0:
            continue
        pos = torch.arange(p, p + n, device="cuda") if positions is None else positions[lo:hi]
        blk, slot = s.place(b, p, p + n)
        check(s.k[blk, :, slot], k_new[lo:hi], kw, eps, offset, pos, inv, interleaved, magnitude, f"k of sequence {b}")
        want_k[blk, :, slot] = s.k[blk, :, slot]
        want_v[blk, :, slot] = v_new[lo:hi]
        if want_q:
            check(out[lo:hi], q0[lo:hi], qw, eps, offset, pos, inv, interleaved, magnitude, f"q of sequence {b}")
    # what must not change stays, bit for bit
    assert torch.equal(s.k.contiguous().view(torch.uint8), want_k.contiguous().view(torch.uint8))
    assert torch.equal(s.v.contiguous().view(torch.uint8), want_v.contiguous().view(torch.uint8))
    if want_q and not in_place:
        assert bool((out[s.rows:] == 5.0).all())
    return out


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d_qk,rot", [(128, 128), (128, 64), (128, 16), (64, 64), (64, 32), (96, 48), (64, 0), (192, 192),
                                      (256, 256), (72, 16), (8, 0), (512, 128)])
def test_pairs_and_parts_of_the_head(api, dtype, interleaved, d_qk, rot):
    step = Step(api, [5, 0, 1000, 77], [3, 40, 1, 0], 8, 2, 4, d_qk, 128, dtype=dtype, pad=2, seed=rot)
    run(api, step.fill(whole=False), rot, interleaved, magnitude=1.0 if rot != 64 else 1.2079)


@pytest.mark.parametrize("dtype,d_qk,rot", [(F32, 2048, 2048), (BF16, 4096, 512), (F32, 1100, 1096), (BF16, 8192, 8192),
                                            (BF16, 520, 16), (F32, 260, 8), (BF16, 1000, 0)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_heads_of_very_many_channels(api, dtype, d_qk, rot, interleaved):
    """More vectors to a head than its lanes hold."""
    step = Step(api, [2, 0], [3, 2], 4, 2, 2, d_qk, 512, dtype=dtype, pad=1, seed=rot)
    run(api, step.fill(whole=False), rot, interleaved, weights="heads")
    step = Step(api, [2, 0], [3, 2], 4, 2, 2, d_qk, 512, dtype=dtype, pad=1, seed=rot)
    run(api, step.fill(whole=False), rot, interleaved, in_place=True)


@pytest.mark.parametrize("weights", ["shared", "heads", "sliced", "keys", "none"])
@pytest.mark.parametrize("dtype,weight_dtype", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("offset", [0.0, 1.0])
def test_weights(api, weights, dtype, weight_dtype, offset):
    step = Step(api, [5, 300], [3, 30], 12, 2, 4, 128, 64, dtype=dtype, pad=2, seed=1)
    run(api, step.fill(whole=False), 64, weights=weights, weight_dtype=weight_dtype, offset=offset)


@pytest.mark.parametrize("heads", [(32, 4, 8), (64, 8, 8), (1, 1, 1), (16, 16, 16), (5, 5, 1), (48, 1, 2)])
@pytest.mark.parametrize("d_qk", [64, 128])
def test_head_counts(api, heads, d_qk):
    step = Step(api, [5, 300], [3, 30], *heads, d_qk, 128, pad=2, seed=1)
    run(api, step.fill(whole=False), d_qk)


@pytest.mark.parametrize("page,layout", [(8, "paged"), (16, "token"), (128, "paged"), (16, "flat"), (24, "paged"), (1, "paged")])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_layouts(api, page, layout, dtype):
    step = Step(api, [30, 0, 129], [7, 140, 1], 8, 2, 4, 64, 64, dtype=dtype, page=page, layout=layout, seed=page, room=3)
    run(api, step.fill(whole=False), 64)


@pytest.mark.parametrize("kw", [dict(in_place=True), dict(fused=True), dict(want_q=False), dict(want_q=False, fused=True)])
def test_ways_to_call(api, kw):
    step = Step(api, [30, 0, 129], [7, 140, 1], 8, 2, 4, 128, 64, seed=2, pad=3)
    run(api, step.fill(whole=False), 128, **kw)


def test_positions_and_another_stream(api):
    step = Step(api, [30, 0, 129], [7, 140, 1], 8, 2, 4, 128, 64, seed=2, pad=3)
    positions = ints([(i * 7919) % 2000003 for i in range(step.total_q)])
    run(api, step.fill(whole=False), 128, positions=positions, stream=torch.cuda.Stream())


@pytest.mark.parametrize("std,eps", [(1e-3, 1e-6), (1e-3, 0.0), (300.0, 1e-5), (1e-12, 1e-6), (1e6, 0.0)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_sizes_of_heads_and_eps(api, std, eps, dtype):
    step = Step(api, [30, 0], [7, 14], 8, 2, 4, 64, 64, seed=2, dtype=dtype)
    run(api, step.fill(whole=False), 64, std=std, eps=eps)


def test_heads_of_zeros(api):
    for eps, want in ((1e-6, 0.0), (0.0, math.nan)):
        step = Step(api, [30], [3], 8, 2, 4, 64, 64, seed=2).fill(whole=False)
        x, k, v = (torch.zeros((3, h, 64), dtype=BF16, device="cuda") for h in (8, 2, 4))
        out = api.diffqkv_norm_rope_append(x, k, v, step.cu, step.cache, None, None, None, eps)
        assert bool((out == 0).all()) if want == 0.0 else bool(torch.isnan(out).all())


def test_a_channel_that_is_not_finite_stays_with_its_head(api):
    step = Step(api, [30], [3], 8, 2, 4, 64, 64, seed=2).fill(whole=False)
    q = torch.ones((3, 8, 64), dtype=BF16, device="cuda")
    q[1, 2, 5] = math.nan
    k, v = (torch.ones((3, h, 64), dtype=BF16, device="cuda") for h in (2, 4))
    out = api.diffqkv_norm_rope_append(q, k, v, step.cu, step.cache, None, None, None, 1e-6)
    bad = torch.isnan(out).all(-1)
    assert bool(bad[1, 2]) and int(bad.sum()) == 1 and int(torch.isnan(out).sum()) == 64


def test_sequences_that_do_not_fit(api):
    step = Step(api, [300, 200, 40], [3, 40, 1], 8, 2, 4, 64, 64, seed=7, pad=1).fill(whole=False)
    step.lens[1] = -1
    out, status = torch.full((step.total_q, 8, 64), 77.0, dtype=BF16, device="cuda"), ints([0])
    before = step.k.clone()
    k, v = (torch.ones((step.total_q, h, 64), dtype=BF16, device="cuda") for h in (2, 4))
    q = torch.ones((step.total_q, 8, 64), dtype=BF16, device="cuda")
    api.diffqkv_norm_rope_append(q, k, v, step.cu, step.cache, None, None, None, 0.0, q_out=out, dev_status=status)
    assert int(status.item()) == 1 << api.ERR_INDEX
    assert bool((out[3:43] == 77.0).all()) and bool((out[44:] == 77.0).all())
    assert bool((out[:3] == 1.0).all()) and bool((out[43] == 1.0).all())
    for b, p, n in ((0, 300, 3), (2, 40, 1)):
        blk, slot = step.place(b, p, p + n)
        before[blk, :, slot] = 1.0
    assert torch.equal(step.k.view(torch.int16), before.view(torch.int16))
    step.table[0, 300 // 16] = 10 ** 6  # no such page: the key is skipped, the query is not
    status.zero_()
    api.diffqkv_norm_rope_append(q, k, v, step.cu, step.cache, None, None, None, 0.0, q_out=out, dev_status=status)
    assert int(status.item()) == 1 << api.ERR_INDEX


def test_offsets_behind_2_31_elements(api):
    """The last page of a large pool, and rows of q and its result behind 2^31 elements."""
    d, n_q = 128, 64
    rows = (1 << 31) // (n_q * d) + 40
    q = torch.zeros((rows, n_q, d), dtype=BF16, device="cuda")
    gen = torch.Generator("cuda").manual_seed(3)
    q[-5:] = torch.randn((5, n_q, d), generator=gen, device="cuda").to(BF16)
    k = torch.ones((rows, 1, d), dtype=BF16, device="cuda")
    pages = (1 << 31) // (128 * d) + 3
    pool = torch.zeros((pages, 1, 128, d), dtype=BF16, device="cuda")
    table = torch.zeros((2, 2), dtype=torch.int32, device="cuda")
    table[1, 0] = pages - 1
    cache = api.KVCache(pool, pool.clone(), ints([0, 0]), 256, page_table=table, page_size=128)
    # one long sequence that does not fit, and five rows at the end
    out = torch.full_like(q, 3.0)
    api.diffqkv_norm_rope_append(q, k, k, ints([0, rows - 5, rows]), cache, None, None, None, 1e-6, q_out=out)
    check(out[-5:], q[-5:], None, 1e-6, 0.0, None, None, False, 1.0, "q")
    assert bool((out[-6] == 3.0).all()) and bool((pool[pages - 1, 0, :5] == 1.0).all())
    assert bool((pool[pages - 1, 0, 5:] == 0).all()) and bool((pool[0] == 0).all())


def test_a_captured_call_replays_with_other_lengths(api):
    cap = 64
    step = Step(api, [30, 40, 50], [10, 10, 10], 8, 2, 4, 64, 64, seed=2, room=60)
    q, k, v = (torch.randn((cap, h, 64), device="cuda").to(BF16) for h in (8, 2, 4))
    w = torch.rand(64, device="cuda").to(BF16)
    inv, _ = api.rope_frequencies(64, 10000.0, device="cuda")
    out, status = torch.zeros_like(q), ints([0])
    call = lambda: api.diffqkv_norm_rope_append(q, k, v, step.cu, step.cache, inv, w, w, 1e-6, q_out=out,  # noqa: E731
                                                dev_status=status)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for past, cu in (([30, 40, 50], [0, 10, 20, 30]), ([1, 0, 20], [0, 0, 40, 64])):
        step.lens.copy_(ints(past))
        step.cu.copy_(ints(cu))
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        for b in range(3):
            lo, hi = cu[b], cu[b + 1]
            if lo < hi and past[b] + hi - lo <= step.max_seqlen:
                pos = torch.arange(past[b], past[b] + hi - lo, device="cuda")
                check(out[lo:hi], q[lo:hi], w, 1e-6, 0.0, pos, inv, False, 1.0, f"q of sequence {b}")
        assert bool((out[cu[-1]:] == 9.0).all())


@pytest.mark.parametrize("d_qk", [64, 128, 520, 1096])
@pytest.mark.parametrize("offset", [0.0, 1.0])
@pytest.mark.parametrize("given", ["neither", "q", "k"])
def test_a_missing_weight_has_no_head_stride(api, d_qk, offset, given):
    """Through the C structure: a stride beside a weight that is NULL changes nothing, for heads that their lanes hold and for
    longer ones."""
    step = Step(api, [5, 300], [3, 30], 12, 2, 4, d_qk, 64, pad=2, seed=1).fill(whole=False)
    gen = torch.Generator("cuda").manual_seed(d_qk)
    q, k, v = (torch.randn((step.total_q, h, d), generator=gen, device="cuda").to(BF16)
               for h, d in ((12, d_qk), (2, d_qk), (4, 64)))
    qw, kw = (torch.randn((h, d_qk), generator=gen, device="cuda").to(BF16) if given == name else None
              for h, name in ((12, "q"), (2, "k")))
    inv = api.rope_frequencies(16, 10000.0, device="cuda")[0]
    pools = step.k.clone(), step.v.clone()
    got = []
    for stray in (0, d_qk, 8 * d_qk):
        step.k.copy_(pools[0])
        step.v.copy_(pools[1])
        strides = [stray if w is None else d_qk for w in (qw, kw)]
        norm = api._pack_norm(*(0 if w is None else w.data_ptr() for w in (qw, kw)), *strides, api.BF16, 1e-6, offset)
        out, status = torch.full_like(q, 5.0), ints([0])
        assert api._raw.diffqkv_norm_rope_append(
            q.data_ptr(), k.data_ptr(), v.data_ptr(), step.cu.data_ptr(), step.total_q, 0, 0, 0, norm,
            api._pack_rope(inv.data_ptr(), 0, 16, False, 1.0), api._cache_bytes(step.cache, 2, 4, d_qk, 64),
            api._pack_shape(2, 12, 2, 4, d_qk, 64, api.BF16, api.BF16, 1.0), out.data_ptr(), status.data_ptr(),
            torch.cuda.current_stream().cuda_stream) == api.OK
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        got.append((out, step.k.clone()))
    pos = torch.arange(5, 8, device="cuda")
    check(got[0][0][:3], q[:3], qw, 1e-6, offset, pos, inv, False, 1.0, "q")
    for out, pool in got[1:]:
        assert torch.equal(out, got[0][0])
        assert torch.equal(pool.view(torch.int16), got[0][1].view(torch.int16))


@pytest.mark.parametrize("d_qk", [64, 128, 2048, 8192])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("end", ["large", "small"])
def test_ends_of_the_range(api, d_qk, dtype, end):
    """Sums of squares within a factor of four of what fp32 holds; heads of 2e-18 without an eps."""
    std = 0.5 * math.sqrt(3.4e38 / d_qk) if end == "large" else 2e-18
    step = Step(api, [3, 0], [4, 3], 4, 2, 2, d_qk, 64, seed=2, dtype=dtype)
    run(api, step.fill(whole=False), 64, std=std, eps=0.0)
