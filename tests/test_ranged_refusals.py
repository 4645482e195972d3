"""What diffqkv_extend_window, diffqkv_extend_shared, diffqkv_norm_rope_append and their Python forms refuse on the host (nothing
is launched, no GPU needed)."""
import ctypes as C
import types

import pytest
import torch

BF16, F32 = torch.bfloat16, torch.float32
A = 4096  # stands for a device pointer: aligned, never read


@pytest.fixture(scope="module")
def api():
    from paper_2501_13629_b200 import build
    build.build()
    from paper_2501_13629_b200 import api as _api
    return _api


def shape(api, **kw):
    d = dict(batch=2, n_q=8, n_k=2, n_v=4, d_qk=64, d_v=64, dtype=BF16, out_dtype=BF16, scale=1.0)
    d.update(kw)
    return api.make_shape(**d)


def cache(api, **kw):
    d = dict(k_cache=A, v_cache=A, k_stride_blk=2048, k_stride_head=1024, k_stride_tok=64, v_stride_blk=4096,
             v_stride_head=1024, v_stride_tok=64, seqlens=A, page_table=A, page_size=16, max_pages_per_seq=4, num_blocks=10,
             max_seqlen=64)
    d.update(kw)
    return api.CacheStruct(**d)


def common_refusals(api, call):
    """What both attention calls share with diffqkv_extend."""
    bad, align, ws, unsup = api.ERR_INVALID_ARG, api.ERR_ALIGNMENT, api.ERR_WORKSPACE, api.ERR_UNSUPPORTED
    assert call(q=None) == bad and call(cu=None) == bad and call(out=None) == bad and call(total=-1) == bad
    assert call(s=shape(api, n_k=3)) == bad and call(s=shape(api, scale=float("nan"))) == bad
    assert call(s=shape(api, d_qk=60)) == unsup and call(s=shape(api, d_v=520)) == unsup
    assert call(c=cache(api, seqlens=None)) == bad and call(c=cache(api, max_seqlen=65)) == bad
    assert call(c=cache(api, k_stride_tok=32)) == bad and call(c=cache(api, k_stride_head=1023)) == align
    assert call(q=A + 8) == align and call(out=A + 2) == align
    assert call(ws=None) == ws and call(ws_bytes=255) == ws and call(ws=A + 16) == align
    assert call(total=0, q=None, out=None) == api.OK and call(s=shape(api, batch=0)) == api.OK


def test_extend_window(api):
    before = api.launch_count()

    def call(s=None, c=None, q=A, cu=A, total=5, window=20, sinks=4, ws=A, ws_bytes=1 << 30, out=A):
        return api._lib.diffqkv_extend_window(q, cu, total, window, sinks, C.byref(c or cache(api)), C.byref(s or shape(api)),
                                              ws, ws_bytes, out, None, None, None)

    common_refusals(api, call)
    assert call(window=0) == api.ERR_INVALID_ARG and call(window=-5) == api.ERR_INVALID_ARG
    assert call(sinks=-1) == api.ERR_INVALID_ARG
    assert call(window=0, total=0) == api.ERR_INVALID_ARG
    need = api.diffqkv_extend_window_workspace_bytes(shape(api), 5)
    assert need >= 256 and need % 256 == 0 and call(ws_bytes=need - 1) == api.ERR_WORKSPACE
    assert api.diffqkv_extend_window_workspace_bytes(shape(api, n_k=3), 5) == 0
    assert api.diffqkv_extend_window_workspace_bytes(shape(api), -1) == 0
    assert api.launch_count() == before


def test_extend_shared(api):
    before = api.launch_count()

    def call(s=None, c=None, q=A, cu=A, total=5, groups=A, lens=A, n=2, ws=A, ws_bytes=1 << 30, out=A):
        prefixes = api.PrefixesStruct(groups, lens, n)
        return api._lib.diffqkv_extend_shared(q, cu, total, C.byref(prefixes), C.byref(c or cache(api)),
                                              C.byref(s or shape(api)), ws, ws_bytes, out, None, None, None)

    common_refusals(api, call)
    bad = api.ERR_INVALID_ARG
    assert call(groups=None) == bad and call(lens=None) == bad and call(n=-1) == bad
    assert call(n=65536) == api.ERR_UNSUPPORTED
    assert call(n=0, groups=None, lens=None, total=0) == api.OK
    assert api._lib.diffqkv_extend_shared(A, A, 5, None, C.byref(cache(api)), C.byref(shape(api)), A, 1 << 30, A, None, None,
                                          None) == bad
    need, plain = api.diffqkv_extend_shared_workspace_bytes(shape(api), 5), api.diffqkv_extend_window_workspace_bytes(shape(api), 5)
    assert need >= plain + 2 * 5 * 8 * (64 + 1) * 4 and need % 256 == 0
    assert call(ws_bytes=need - 1) == api.ERR_WORKSPACE
    # a step without tensor cores needs a length for every sequence
    f32 = shape(api, dtype=F32, batch=1000)
    assert api.diffqkv_extend_shared_workspace_bytes(f32, 5) >= api.diffqkv_extend_workspace_bytes(f32, 5) + 4000
    assert api.diffqkv_extend_shared_workspace_bytes(shape(api, n_k=3), 5) == 0
    assert api.diffqkv_extend_shared_workspace_bytes(shape(api), -1) == 0
    assert api.launch_count() == before


def test_norm_rope_append(api):
    before = api.launch_count()

    def call(s=None, c=None, q=A, k=A, v=A, cu=A, total=5, strides=(0, 0, 0), out=A, norm=None, rope=None, **kw):
        n = dict(q_weight=A, k_weight=A, q_head_stride=0, k_head_stride=0, weight_dtype=api.BF16, eps=1e-6, weight_offset=0.0)
        n.update(kw)
        r = dict(inv_freq=A, positions=None, rot_dim=64, interleaved=0, magnitude=1.0)
        r.update(rope or {})
        return api._lib.diffqkv_norm_rope_append(q, k, v, cu, total, *strides, C.byref(api.QkNormStruct(**n)) if norm is None else
                                                 norm[0], C.byref(api.RopeStruct(**r)), C.byref(c or cache(api)),
                                                 C.byref(s or shape(api)), out, None, None)

    bad, align, unsup = api.ERR_INVALID_ARG, api.ERR_ALIGNMENT, api.ERR_UNSUPPORTED
    assert call(k=None) == bad and call(v=None) == bad and call(cu=None) == bad and call(out=None) == bad
    assert call(total=-1) == bad and call(norm=[None]) == bad
    assert call(rope=dict(rot_dim=80)) == bad and call(rope=dict(rot_dim=24)) == unsup
    assert call(rope=dict(inv_freq=None)) == bad and call(rope=dict(magnitude=float("nan"))) == bad
    assert call(strides=(511, 0, 0)) == bad and call(strides=(516, 0, 0)) == align and call(strides=(520, 0, 0)) == bad
    assert call(k=A + 2) == align and call(c=cache(api, k_cache=None)) == bad
    assert call(eps=-1e-6) == bad and call(eps=float("nan")) == bad and call(weight_offset=float("nan")) == bad
    assert call(weight_dtype=7) == bad
    f32_cache = cache(api, k_stride_tok=64)
    assert call(s=shape(api, dtype=F32), c=f32_cache, weight_dtype=api.BF16) == unsup
    assert call(q_weight=A + 8) == align and call(k_weight=A + 2) == align
    assert call(q_head_stride=56) == bad and call(k_head_stride=-64) == bad and call(q_head_stride=68) == align
    assert call(k_head_stride=66, weight_dtype=api.F32) == align
    assert call(total=0, k=None) == api.OK and call(s=shape(api, batch=0)) == api.OK
    assert api.launch_count() == before


# ---- the Python forms

STREAM = types.SimpleNamespace(cuda_stream=0)


@pytest.fixture()
def recorded(api, monkeypatch):
    """The wrappers over tensors on the host; calls that get as far as the library are recorded, not made."""
    calls = []
    monkeypatch.setattr(api, "_device_of", lambda *t: 0)
    for name in ("diffqkv_extend_window", "diffqkv_extend_shared", "diffqkv_norm_rope_append"):
        monkeypatch.setattr(api._raw, name, lambda *args: (calls.append(args), 0)[1])
    monkeypatch.setattr(api, "_fresh", lambda shape, dtype, device, stream: torch.empty(shape, dtype=dtype))
    return calls


def z(*shape, dtype=BF16):
    return torch.zeros(shape, dtype=dtype)


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def kv(api):
    return api.KVCache(k=z(6, 2, 16, 64), v=z(6, 4, 16, 64), seqlens=ints(2), max_seqlen=48, page_table=ints(2, 3), page_size=16)


def refused(calls, call):
    before = len(calls)
    with pytest.raises((ValueError, AssertionError)):
        call()
    assert len(calls) == before


def made(calls, call):
    before = len(calls)
    call()
    assert len(calls) == before + 1
    return calls[-1]


def test_wrappers_of_the_attention_calls(api, recorded):
    window = lambda q=z(5, 8, 64), cu=ints(3), **kw: api.diffqkv_extend_window(  # noqa: E731
        q, cu, kv(api), 2, 4, 0.125, 16, sinks=2, stream=STREAM, **kw)
    assert made(recorded, window)[2:5] == (5, 16, 2)
    far = lambda window, sinks: made(recorded, lambda: api.diffqkv_extend_window(  # noqa: E731
        z(5, 8, 64), ints(3), kv(api), 2, 4, 0.125, window, sinks=sinks, stream=STREAM))[3:5]
    assert far(2 ** 32 + 5, 2 ** 63 - 1) == (2 ** 31 - 1, 2 ** 31 - 1) and far(-2 ** 32 + 5, -2 ** 32) == (-1, -1)
    refused(recorded, lambda: window(q=z(5, 8, 32)))
    refused(recorded, lambda: window(q=z(5, 8, 64, dtype=F32)))
    refused(recorded, lambda: window(cu=ints(4)))
    refused(recorded, lambda: window(out=z(5, 8, 32)))
    refused(recorded, lambda: window(lse=z(5, 8)))
    shared = lambda groups=ints(3), lens=ints(2), **kw: api.diffqkv_extend_shared(  # noqa: E731
        z(5, 8, 64), ints(3), kv(api), groups, lens, 2, 4, 0.125, stream=STREAM, **kw)
    groups, lens = ints(3), ints(2)
    args = made(recorded, lambda: shared(groups, lens))
    packed = api.PrefixesStruct.from_buffer_copy(args[3])
    assert (packed.cu_seqs, packed.lens, packed.num_groups) == (groups.data_ptr(), lens.data_ptr(), 2)
    refused(recorded, lambda: shared(groups=ints(2)))
    refused(recorded, lambda: shared(lens=torch.zeros(2, dtype=torch.int64)))
    refused(recorded, lambda: shared(lens=ints(4)[::2]))
    refused(recorded, lambda: shared(out=z(4, 8, 64)))


def test_wrapper_of_the_norms(api, recorded):
    norm = lambda qw=z(64), kw=z(64), q=z(5, 8, 64), **more: api.diffqkv_norm_rope_append(  # noqa: E731
        q, z(5, 2, 64), z(5, 4, 64), ints(3), kv(api), None, qw, kw, 1e-6, stream=STREAM, **more)
    unpack = lambda args: api.QkNormStruct.from_buffer_copy(args[8])  # noqa: E731
    qw, kw = z(8, 64), z(2, 192)[:, 64:128]
    s = unpack(made(recorded, lambda: norm(qw, kw, weight_offset=1.0)))
    assert (s.q_weight, s.k_weight, s.q_head_stride, s.k_head_stride) == (qw.data_ptr(), kw.data_ptr(), 64, 192)
    assert s.weight_dtype == api.BF16 and s.weight_offset == 1.0 and abs(s.eps - 1e-6) < 1e-12
    s = unpack(made(recorded, lambda: norm(None, z(64, dtype=F32))))
    assert s.q_weight is None and s.weight_dtype == api.F32 and s.k_head_stride == 0
    assert unpack(made(recorded, lambda: norm(None, None))).k_weight is None
    assert unpack(made(recorded, lambda: norm(z(1, 64).expand(8, 64)))).q_head_stride == 0
    made(recorded, lambda: norm(None, q=None))
    refused(recorded, lambda: norm(z(32)))
    refused(recorded, lambda: norm(z(4, 64)))
    refused(recorded, lambda: norm(z(64, dtype=F32)))  # not k_weight's type
    refused(recorded, lambda: norm(z(128)[::2]))
    refused(recorded, lambda: norm(torch.as_strided(z(600), (8, 64), (32, 1))))
    refused(recorded, lambda: norm(kw=z(8, 64)))
    refused(recorded, lambda: norm(q_out=z(5, 8, 32)))


def test_calls_on_the_host_are_refused(api):
    """The tensors have to be on the GPU."""
    before = api.launch_count()
    with pytest.raises(ValueError):
        api.diffqkv_extend_window(z(5, 8, 64), ints(3), kv(api), 2, 4, 0.125, 16)
    with pytest.raises(ValueError):
        api.diffqkv_extend_shared(z(5, 8, 64), ints(3), kv(api), ints(3), ints(2), 2, 4, 0.125)
    with pytest.raises(ValueError):
        api.diffqkv_norm_rope_append(z(5, 8, 64), z(5, 2, 64), z(5, 4, 64), ints(3), kv(api), None, None, None, 1e-6)
    assert api.launch_count() == before


def test_the_queries_weight_where_there_are_no_queries(api, recorded):
    """A step that only writes keys may be given the layer's two weights all the same."""
    for qw in (z(64), z(8, 64), z(1, 64).expand(8, 64), None):
        args = made(recorded, lambda: api.diffqkv_norm_rope_append(None, z(5, 2, 64), z(5, 4, 64), ints(3), kv(api), None, qw,
                                                                   z(64), 1e-6, stream=STREAM))
        s = api.QkNormStruct.from_buffer_copy(args[8])
        assert s.q_weight is None and s.q_head_stride == 0 and s.k_weight is not None and s.weight_dtype == api.BF16
        assert args[0] in (None, 0)
    args = made(recorded, lambda: api.diffqkv_norm_rope_append(None, z(5, 2, 64), z(5, 4, 64), ints(3), kv(api), None,
                                                               z(8, 64, dtype=F32), None, 1e-6, stream=STREAM))
    assert api.QkNormStruct.from_buffer_copy(args[8]).q_weight is None
