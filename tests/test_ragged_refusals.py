"""What the ragged-batch entry points refuse on the host (nothing is launched, no GPU needed), and the frequency tables."""
import ctypes as C
import math

import pytest
import torch


@pytest.fixture(scope="module")
def api():
    from paper_2501_13629_b200 import build
    build.build()
    from paper_2501_13629_b200 import api as _api
    return _api


A = 4096  # stands for a device pointer: aligned, never read


def shape(api, **kw):
    d = dict(batch=2, n_q=8, n_k=2, n_v=4, d_qk=64, d_v=64, dtype=torch.bfloat16, out_dtype=torch.bfloat16, scale=1.0)
    d.update(kw)
    return api.make_shape(**d)


def cache(api, **kw):
    d = dict(k_cache=A, v_cache=A, k_stride_blk=2048, k_stride_head=1024, k_stride_tok=64, v_stride_blk=4096,
             v_stride_head=1024, v_stride_tok=64, seqlens=A, page_table=A, page_size=16, max_pages_per_seq=4, num_blocks=10,
             max_seqlen=64)
    d.update(kw)
    return api.CacheStruct(**d)


def pages(api, **kw):
    d = dict(page_table=A, seqlens=A, ref_counts=A, num_seqs=2, max_pages_per_seq=4, num_pages=10, page_size=16)
    d.update(kw)
    return api.PagesStruct(**d)


def extend(api, s=None, c=None, q=A, cu=A, total=5, ws=A, ws_bytes=1 << 30, out=A):
    return api._lib.diffqkv_extend(q, cu, total, C.byref(c or cache(api)), C.byref(s or shape(api)), ws, ws_bytes, out, None,
                                   None, None)


def test_extend_refusals(api):
    before = api.launch_count()
    bad, align, ws, unsup = api.ERR_INVALID_ARG, api.ERR_ALIGNMENT, api.ERR_WORKSPACE, api.ERR_UNSUPPORTED
    assert extend(api, q=None) == bad and extend(api, cu=None) == bad and extend(api, out=None) == bad
    assert extend(api, total=-1) == bad
    assert extend(api, s=shape(api, n_k=3)) == bad and extend(api, s=shape(api, scale=float("nan"))) == bad
    assert extend(api, s=shape(api, d_qk=60)) == unsup and extend(api, s=shape(api, d_v=520)) == unsup
    assert extend(api, c=cache(api, seqlens=None)) == bad and extend(api, c=cache(api, max_seqlen=65)) == bad
    assert extend(api, c=cache(api, k_stride_tok=32)) == bad and extend(api, c=cache(api, k_stride_head=1023)) == align
    assert extend(api, q=A + 8) == align and extend(api, out=A + 2) == align
    assert extend(api, ws=None) == ws and extend(api, ws_bytes=255) == ws and extend(api, ws=A + 16) == align
    assert extend(api, total=0, q=None, out=None) == api.OK and extend(api, s=shape(api, batch=0)) == api.OK
    assert api.launch_count() == before
    need = api.diffqkv_extend_workspace_bytes(shape(api), 5)
    assert need >= 256 and need % 256 == 0
    assert api.diffqkv_extend_workspace_bytes(shape(api, n_k=3), 5) == 0
    assert api.diffqkv_extend_workspace_bytes(shape(api), -1) == 0


def test_rope_append_refusals(api):
    before = api.launch_count()

    def call(s=None, c=None, q=A, k=A, v=A, cu=A, total=5, strides=(0, 0, 0), out=A, **kw):
        r = dict(inv_freq=A, positions=None, rot_dim=64, interleaved=0, magnitude=1.0)
        r.update(kw)
        rope = api.RopeStruct(**r)
        return api._lib.diffqkv_rope_append(q, k, v, cu, total, *strides, C.byref(rope), C.byref(c or cache(api)),
                                            C.byref(s or shape(api)), out, None, None)

    bad, align, unsup = api.ERR_INVALID_ARG, api.ERR_ALIGNMENT, api.ERR_UNSUPPORTED
    assert call(k=None) == bad and call(v=None) == bad and call(cu=None) == bad and call(out=None) == bad
    assert call(total=-1) == bad and call(rot_dim=80) == bad and call(rot_dim=-16) == bad and call(inv_freq=None) == bad
    assert call(rot_dim=24) == unsup and call(rot_dim=8) == unsup and call(magnitude=float("nan")) == bad
    assert call(s=shape(api, dtype=torch.float32), c=cache(api), rot_dim=12) == unsup
    assert call(inv_freq=A + 4) == align and call(k=A + 2) == align
    assert call(strides=(511, 0, 0)) == bad and call(strides=(516, 0, 0)) == align
    assert call(strides=(0, 0, 252)) == bad
    assert call(strides=(520, 0, 0), out=A) == bad  # in place needs dense rows
    assert call(c=cache(api, k_cache=None)) == bad
    assert call(total=0, k=None) == api.OK and call(s=shape(api, batch=0)) == api.OK
    assert api.launch_count() == before


def test_pages_refusals(api):
    before = api.launch_count()
    lib, bad, ws, align = api._lib, api.ERR_INVALID_ARG, api.ERR_WORKSPACE, api.ERR_ALIGNMENT
    free = lambda g, ids=A, n=1: lib.diffqkv_pages_free(ids, None, n, C.byref(g), None, None)  # noqa: E731
    for field in ("page_table", "seqlens", "ref_counts"):
        assert free(pages(api, **{field: None})) == bad
    for field in ("max_pages_per_seq", "num_pages", "page_size"):
        assert free(pages(api, **{field: 0})) == bad
    assert free(pages(api, num_pages=(1 << 20) + 1)) == api.ERR_UNSUPPORTED
    assert free(pages(api, num_seqs=65536)) == api.ERR_UNSUPPORTED
    assert free(pages(api), ids=None) == bad and free(pages(api), n=-1) == bad and free(pages(api), ids=None, n=0) == api.OK

    def fork(g=None, parents=A, n=1, space=A, size=1 << 20):
        return lib.diffqkv_pages_fork(parents, A, n, C.byref(g or pages(api)), space, size, None, None)

    assert fork(parents=None) == bad and fork(n=-1) == bad and fork(parents=None, n=0) == api.OK
    assert fork(space=None) == ws and fork(size=16) == ws and fork(space=A + 8) == align
    assert lib.diffqkv_pages_fork_workspace_bytes(C.byref(pages(api)), -1) == 0
    assert lib.diffqkv_pages_fork_workspace_bytes(C.byref(pages(api)), 3) >= 3 * 5 * 4

    def reserve(g=None, c=None, s=None, cu=A, space=A, size=1 << 20):
        return lib.diffqkv_pages_reserve(cu, C.byref(g or pages(api)), C.byref(c or cache(api)), C.byref(s or shape(api)),
                                         None, space, size, None, None)

    assert reserve(cu=None) == bad and reserve(c=cache(api, page_size=32)) == bad
    assert reserve(c=cache(api, num_blocks=9)) == bad and reserve(c=cache(api, v_cache=None)) == bad
    assert reserve(c=cache(api, v_stride_tok=66)) == align and reserve(c=cache(api, k_cache=A + 8)) == align
    assert reserve(s=shape(api, d_qk=60)) == api.ERR_UNSUPPORTED
    assert reserve(space=None) == ws and reserve(size=100) == ws and reserve(g=pages(api, num_seqs=0)) == api.OK

    def copy(src=A, n=1, a=None, b=None):
        return lib.diffqkv_pages_copy(src, A, n, C.byref(a or cache(api)), C.byref(b or cache(api)), C.byref(shape(api)),
                                      None, None)

    assert copy(src=None) == bad and copy(n=-1) == bad and copy(src=None, n=0) == api.OK
    assert copy(b=cache(api, page_size=8)) == bad and copy(a=cache(api, page_size=0), b=cache(api, page_size=0)) == bad

    def compact(table=A, refs=A, c=None, size=1 << 20):
        return lib.diffqkv_pages_compact(C.byref(pages(api)), C.byref(c or cache(api)), C.byref(shape(api)), table, refs,
                                         None, A, size, None, None)

    assert compact(table=None) == bad and compact(refs=None) == bad and compact(c=cache(api, num_blocks=11)) == bad
    assert compact(size=300) == ws
    assert api.launch_count() == before


def test_tensors_elsewhere_are_refused(api):
    """The wrappers take CUDA tensors only: a host pointer would be read by a kernel."""
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    c = api.KVCache(z(4, 2, 16, 64), z(4, 4, 16, 64), i(1), 32, page_table=i(1, 2), page_size=16)
    for call in (lambda: api.diffqkv_extend(z(1, 8, 64), i(2), c, 2, 4, 1.0),
                 lambda: api.diffqkv_rope_append(z(1, 8, 64), z(1, 2, 64), z(1, 4, 64), i(2), c, None),
                 lambda: api.diffqkv_pages_free(i(1), c, i(4)),
                 lambda: api.diffqkv_pages_fork(i(1), i(1), c, i(4)),
                 lambda: api.diffqkv_pages_reserve(i(2), c, i(4), 2, 4),
                 lambda: api.diffqkv_pages_copy(i(1), i(1), c, 2, 4),
                 lambda: api.diffqkv_pages_compact(c, i(4), 2, 4)):
        with pytest.raises(ValueError):
            call()


# ---- frequency tables, against the formulas

def table(rot, theta):
    return [theta ** (-2.0 * i / rot) for i in range(rot // 2)]


@pytest.mark.parametrize("rot,theta", [(2, 10000.0), (64, 50000.0), (128, 500000.0), (96, 1e6)])
def test_frequencies(api, rot, theta):
    def same(got, want, magnitude=1.0):
        assert got[0].dtype == torch.float64 and got[0].numel() == rot // 2
        # pow and the divisions are good to a few steps of fp64
        assert all(abs(a - b) <= 1e-14 * b for a, b in zip(got[0].tolist(), want))
        assert abs(got[1] - magnitude) <= 2.0 ** -23 * magnitude

    f = table(rot, theta)
    same(api.rope_frequencies(rot, theta), f)
    same(api.rope_frequencies(rot, theta, "linear", factor=4.0), [x / 4.0 for x in f])
    if rot > 2:
        same(api.rope_frequencies(rot, theta, "ntk", factor=8.0), table(rot, theta * 8.0 ** (rot / (rot - 2))))
    L, s, fast, slow = 4096.0, 16.0, 32.0, 1.0
    c = lambda r: rot * math.log(L / (2 * math.pi * r)) / (2 * math.log(theta))  # noqa: E731
    lo, hi = max(math.floor(c(fast)), 0), min(math.ceil(c(slow)), rot - 1)
    hi = hi if hi > lo else lo + 1e-3
    g = [min(max((i - lo) / (hi - lo), 0.0), 1.0) for i in range(rot // 2)]
    same(api.rope_frequencies(rot, theta, "yarn", factor=s, original_length=L, fast=fast, slow=slow),
         [x * (1 - w) + x / s * w for x, w in zip(f, g)], 0.1 * math.log(s) + 1)
    L, s, fast, slow = 8192.0, 8.0, 4.0, 1.0
    want = []
    for x in f:
        wave = 2 * math.pi / x
        t = (L / wave - slow) / (fast - slow)
        want.append(x if wave < L / fast else x / s if wave > L / slow else (1 - t) * x / s + t * x)
    same(api.rope_frequencies(rot, theta, "bands", factor=s, original_length=L, fast=fast, slow=slow), want)


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=-4), dict(theta=1.0), dict(theta=math.nan),
                                dict(scaling="linear", factor=0.5), dict(scaling="ntk", factor=2.0, rot_dim=2),
                                dict(scaling="yarn", factor=2.0), dict(scaling="yarn", factor=math.inf),
                                dict(scaling="bands", factor=2.0, original_length=100.0, fast=1.0, slow=2.0)])
def test_frequency_refusals(api, kw):
    args = dict(rot_dim=64, theta=10000.0)
    args.update(kw)
    with pytest.raises(api.DiffQKVError) as e:
        api.rope_frequencies(**args)
    assert e.value.status == api.ERR_INVALID_ARG
    assert api._lib.diffqkv_rope_frequencies(64, 10000.0, 9, 1.0, 0.0, 0.0, 0.0, (C.c_double * 32)(), None) == e.value.status


def test_new_status_has_a_text(api):
    assert api.status_string(api.ERR_PAGES) not in {api.status_string(i) for i in range(8)}
