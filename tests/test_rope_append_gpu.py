"""diffqkv_rope_append: rotation of ragged q and k rows and their write into the cache, against float64."""
import math

import pytest
import torch

from ragged import BF16, F32, HALF_STEP, Step, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2501_13629_b200 import api as _api
    return _api


def turned64(x, pos, inv_freq, interleaved, magnitude):
    """x [rows, heads, d] at positions pos [rows]: float64."""
    y = x.double().clone()
    if inv_freq is None:
        return y
    half = inv_freq.numel()
    angle = torch.outer(pos.double(), inv_freq)[:, None]
    i = torch.arange(half, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    u, v = x[..., a].double(), x[..., b].double()
    y[..., a] = magnitude * (u * angle.cos() - v * angle.sin())
    y[..., b] = magnitude * (v * angle.cos() + u * angle.sin())
    return y


def check(out, ref, x, inv_freq, interleaved, magnitude, what):
    """cos and sin are off by 4 steps of fp32 at most (half a step for the reduced angle of up to pi, two for sincosf, one
    for the magnitude), each product and the difference by one more: 8 2^-23 (|u| + |v|) magnitude; then one rounding.
    Channels that are not rotated are copied."""
    if inv_freq is None:
        assert torch.equal(out, x), what
        return
    rot, half = 2 * inv_freq.numel(), inv_freq.numel()
    big = torch.zeros_like(ref)
    i = torch.arange(half, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    s = (x[..., a].double().abs() + x[..., b].double().abs()) * magnitude
    big[..., a], big[..., b] = s, s
    loss = 8 * 2.0 ** -23 * big
    bound = loss + HALF_STEP[out.dtype] * (ref.abs() + loss) + 1e-38
    err = (out.double() - ref).abs()
    assert bool((err <= bound)[..., :rot].all()), f"{what}: {float((err / bound)[..., :rot].max()):.2f} times the bound"
    assert torch.equal(out[..., rot:], x[..., rot:]), what


def run(api, step, rot, interleaved=False, magnitude=1.0, theta=500000.0, positions=None, in_place=False, fused=False,
        want_q=True):
    s = step
    inv = None if rot == 0 else api.rope_frequencies(rot, theta, device="cuda")[0]
    k_new = torch.full((s.total_q, s.n_k, s.d_qk), math.nan, dtype=s.dtype, device="cuda")
    v_new = torch.full((s.total_q, s.n_v, s.d_v), math.nan, dtype=s.dtype, device="cuda")
    for b, p in enumerate(s.past):
        k_new[s.cu_host[b]:s.cu_host[b + 1]] = s.k_tok[b][p:]
        v_new[s.cu_host[b]:s.cu_host[b + 1]] = s.v_tok[b][p:]
    q = s.q.clone()
    if fused:  # slices of one projection's output
        both = torch.cat([x.reshape(s.total_q, -1) for x in (q, k_new, v_new)], 1)
        cut = [s.n_q * s.d_qk, (s.n_q + s.n_k) * s.d_qk]
        q = both[:, :cut[0]].unflatten(1, (s.n_q, s.d_qk))
        k_new = both[:, cut[0]:cut[1]].unflatten(1, (s.n_k, s.d_qk))
        v_new = both[:, cut[1]:].unflatten(1, (s.n_v, s.d_v))
    out = q if in_place else torch.full((s.total_q, s.n_q, s.d_qk), 5.0, dtype=s.dtype, device="cuda")
    before_k, before_v, q0 = s.k.clone(), s.v.clone(), q.clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.diffqkv_rope_append(q if want_q else None, k_new, v_new, s.cu, s.cache, inv, interleaved=interleaved,
                            magnitude=magnitude, positions=positions, q_out=out if want_q else None, dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    want_k, want_v = before_k, before_v  # what must not change stays, bit for bit
    for b, (p, n) in enumerate(zip(s.past, s.new)):
        lo, hi = s.cu_host[b], s.cu_host[b + 1]
        if n == 0:
            continue
        pos = torch.arange(p, p + n, device="cuda") if positions is None else positions[lo:hi]
        blk, slot = s.place(b, p, p + n)
        ref = turned64(k_new[lo:hi], pos, inv, interleaved, magnitude)
        check(s.k[blk, :, slot], ref, k_new[lo:hi], inv, interleaved, magnitude, f"k of sequence {b}")
        want_k[blk, :, slot] = s.k[blk, :, slot]
        want_v[blk, :, slot] = v_new[lo:hi]
        if want_q:
            check(out[lo:hi], turned64(q0[lo:hi], pos, inv, interleaved, magnitude), q0[lo:hi], inv, interleaved, magnitude,
                  f"q of sequence {b}")
    assert torch.equal(s.k.contiguous().view(torch.uint8), want_k.contiguous().view(torch.uint8))
    assert torch.equal(s.v.contiguous().view(torch.uint8), want_v.contiguous().view(torch.uint8))
    if want_q and not in_place:
        assert bool((out[s.rows:] == 5.0).all())
    return out


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d_qk,rot", [(128, 128), (128, 64), (128, 16), (64, 64), (64, 32), (96, 48), (64, 0), (192, 192)])
def test_pairs_and_parts_of_the_head(api, dtype, interleaved, d_qk, rot):
    step = Step(api, [5, 0, 1000, 77], [3, 40, 1, 0], 8, 2, 4, d_qk, 128, dtype=dtype, pad=2, seed=rot)
    run(api, step.fill(whole=False), rot, interleaved, magnitude=1.0 if rot != 64 else 1.2079)


@pytest.mark.parametrize("dtype,d_qk,rot", [(F32, 2048, 2048), (BF16, 4096, 512), (F32, 1100, 1096), (BF16, 8192, 8192)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_heads_of_very_many_channels(api, dtype, d_qk, rot, interleaved):
    """More vectors to a head than a block has threads."""
    step = Step(api, [2, 0], [3, 2], 2, 1, 2, d_qk, 512, dtype=dtype, pad=1, seed=rot)
    run(api, step.fill(whole=False), rot, interleaved)


@pytest.mark.parametrize("layout,page", [("paged", 16), ("token", 16), ("flat", 16), ("paged", 24), ("paged", 1),
                                         ("paged", 256)])
def test_layouts(api, layout, page):
    step = Step(api, [30, 0, 511], [50, 1, 17], 6, 2, 3, 64, 64, page=page, layout=layout, seed=page, room=9)
    run(api, step.fill(whole=False), 64)


@pytest.mark.parametrize("base", [0, 100_000, 1_000_000, 16_777_217, 2_000_000_000])
def test_far_positions(api, base):
    """Angles of 10^5 radians and more keep their fraction; negative positions turn the other way."""
    step = Step(api, [3, 0], [60, 4], 4, 2, 2, 128, 64, dtype=F32, seed=1)
    pos = base + torch.arange(64, device="cuda", dtype=torch.int32) * 13
    run(api, step.fill(whole=False), 128, positions=pos, theta=10000.0)
    step = Step(api, [3, 0], [60, 4], 4, 2, 2, 128, 64, dtype=F32, seed=2)
    run(api, step.fill(whole=False), 128, positions=-pos, interleaved=True)


@pytest.mark.parametrize("kw", [dict(in_place=True), dict(fused=True), dict(want_q=False), dict(fused=True, want_q=False)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_call_forms(api, kw, dtype):
    step = Step(api, [30, 2, 511], [50, 1, 17], 8, 2, 4, 64, 128, dtype=dtype, seed=7)
    run(api, step.fill(whole=False), 64, **kw)


def test_many_sequences(api):
    step = Step(api, [i % 50 for i in range(900)], [(i * 7) % 3 for i in range(900)], 4, 2, 2, 64, 64, seed=3, pad=4)
    run(api, step.fill(whole=False), 32)


def test_turn_is_relative(api):
    """Scores depend on the distance alone: moving every position by the same amount changes no inner product."""
    q, k = (torch.randn((16, 1, 128), device="cuda", generator=torch.Generator("cuda").manual_seed(i)) for i in (1, 2))
    inv = api.rope_frequencies(128, 10000.0, device="cuda")[0]
    scores = []
    for base in (0, 70001):
        k_pool, v_pool = torch.zeros((1, 1, 16, 128), device="cuda"), torch.zeros((1, 1, 16, 64), device="cuda")
        cache = api.KVCache(k_pool, v_pool, ints([0]), 16)
        pos = base + torch.arange(16, device="cuda", dtype=torch.int32)
        out = api.diffqkv_rope_append(q, k, torch.zeros((16, 1, 64), device="cuda"), ints([0, 16]), cache, inv,
                                      positions=pos)
        scores.append(out[:, 0].double() @ k_pool[0, 0].double().T)
    # two turned vectors, each off by 8 2^-23 per pair: 16 2^-23 |q| |k| of the inner product, for both sides
    assert float((scores[0] - scores[1]).abs().max()) <= 64 * 2.0 ** -23 * float(q.norm(dim=2).max() * k.norm(dim=2).max())


def test_rows_that_do_not_fit_and_bad_pages(api):
    step = Step(api, [30, 2], [20, 3], 4, 2, 2, 64, 64, seed=5).fill(whole=False)
    inv = api.rope_frequencies(64, 10000.0, device="cuda")[0]
    k_new, v_new = torch.ones((23, 2, 64), dtype=BF16, device="cuda"), torch.ones((23, 2, 64), dtype=BF16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call(lens, table, cu=step.cu):
        status.zero_()
        cache = api.KVCache(step.k, step.v, ints(lens), step.max_seqlen, page_table=table, page_size=16)
        out = torch.full((23, 4, 64), 5.0, dtype=BF16, device="cuda")
        api.diffqkv_rope_append(step.q, k_new, v_new, cu, cache, inv, q_out=out, dev_status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == 1 << api.ERR_INDEX
        return out

    before = step.k.clone()
    out = call([step.max_seqlen - 19, 2], step.table)
    assert bool((out[:20] == 5.0).all()) and not bool((out[20:] == 5.0).any())
    blk, slot = step.place(1, 2, 5)
    before[blk, :, slot] = step.k[blk, :, slot]
    assert torch.equal(step.k.view(torch.int16), before.view(torch.int16))
    for bad in (-1, 10 ** 6):
        table = step.table.clone()
        table[0, 2] = bad
        out = call([30, 2], table)
        assert not bool((out == 5.0).all(-1).any())  # the queries are turned all the same
    for cu in ([0, 20, 19], [0, 20, 24], [0, -3, 23]):
        call([30, 2], step.table, ints(cu))
