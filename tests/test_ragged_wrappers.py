"""What the Python forms of the ragged-batch calls refuse before the library is called (no GPU: the tensors lie on the host,
and a call that gets as far as the library is recorded, not made)."""
import ctypes as C
import types

import pytest
import torch

BF16 = torch.bfloat16


@pytest.fixture()
def api(monkeypatch):
    from paper_2501_13629_b200 import build
    build.build()
    from paper_2501_13629_b200 import api as _api
    monkeypatch.setattr(_api, "_device_of", lambda *t: 0)
    _api_calls = []
    for name in ("diffqkv_extend", "diffqkv_rope_append", "diffqkv_pages_free", "diffqkv_pages_fork", "diffqkv_pages_reserve",
                 "diffqkv_pages_copy", "diffqkv_pages_compact"):
        monkeypatch.setattr(_api._raw, name, lambda *args, name=name: (_api_calls.append((name, args)), 0)[1])
    _api_calls.clear()
    monkeypatch.setattr(_api, "test_calls", _api_calls, raising=False)
    monkeypatch.setattr(_api, "_fresh", lambda shape, dtype, device, stream: torch.empty(shape, dtype=dtype))
    return _api


STREAM = types.SimpleNamespace(cuda_stream=0)


def z(*shape, dtype=BF16):
    return torch.zeros(shape, dtype=dtype)


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def cache(api, **kw):
    """Two sequences, 2 K heads and 4 V heads of 64 channels, pages of 16 tokens."""
    d = dict(k=z(6, 2, 16, 64), v=z(6, 4, 16, 64), seqlens=ints(2), max_seqlen=48, page_table=ints(2, 3), page_size=16)
    d.update(kw)
    return api.KVCache(**d)


def rope(api, q=None, k=None, v=None, c=None, **kw):
    return api.diffqkv_rope_append(z(5, 8, 64) if q is None else q, z(5, 2, 64) if k is None else k,
                                   z(5, 4, 64) if v is None else v, ints(3), c or cache(api), None, stream=STREAM, **kw)


def refused(api, call):
    before = len(api.test_calls)
    with pytest.raises((ValueError, AssertionError)):
        call()
    assert len(api.test_calls) == before


def made(api, call):
    before = len(api.test_calls)
    call()
    assert len(api.test_calls) == before + 1
    return api.test_calls[-1][1]


def test_broadcast_rows_are_refused(api):
    """A row stride of 0 means dense to the library: one row expanded to several would be read behind its end."""
    made(api, lambda: rope(api))
    refused(api, lambda: rope(api, q=z(1, 8, 64).expand(5, 8, 64)))
    refused(api, lambda: rope(api, k=z(1, 2, 64).expand(5, 2, 64)))
    refused(api, lambda: rope(api, v=z(1, 4, 64).expand(5, 4, 64)))
    refused(api, lambda: rope(api, k=torch.as_strided(z(600), (5, 2, 64), (64, 64, 1))))  # rows that overlap
    fused = z(5, 14 * 64)
    args = made(api, lambda: rope(api, q=fused[:, :512].unflatten(1, (8, 64)), k=fused[:, 512:640].unflatten(1, (2, 64)),
                                  v=fused[:, 640:].unflatten(1, (4, 64))))
    assert args[5:8] == (896, 896, 896)
    one = lambda h: z(1, h, 64).expand(1, h, 64)  # noqa: E731
    assert made(api, lambda: rope(api, q=one(8), k=one(2), v=one(4)))[5:8] == (0, 0, 0)


def extend(api, c=None, q=None, n_k=2, n_v=4, **kw):
    q = z(5, 8, 64) if q is None else q
    return api.diffqkv_extend(q, ints(3), c or cache(api), n_k, n_v, 0.125, stream=STREAM, **kw)


def test_heads_and_channels_are_the_pools(api):
    """More heads than a pool has would be written behind a page; keys of another width are other keys."""
    made(api, lambda: rope(api))
    refused(api, lambda: rope(api, k=z(5, 4, 64)))
    refused(api, lambda: rope(api, v=z(5, 8, 64)))
    refused(api, lambda: rope(api, q=z(5, 8, 32), k=z(5, 2, 32)))
    refused(api, lambda: rope(api, v=z(5, 4, 32)))
    made(api, lambda: extend(api))
    refused(api, lambda: extend(api, q=z(5, 8, 32)))
    refused(api, lambda: extend(api, n_k=4))
    refused(api, lambda: extend(api, n_v=8))
    for heads in (dict(n_k=1, n_v=4), dict(n_k=4, n_v=4), dict(n_k=2, n_v=2), dict(n_k=2, n_v=8)):
        refused(api, lambda: api.diffqkv_pages_reserve(ints(3), cache(api), ints(6), stream=STREAM, **heads))
        refused(api, lambda: api.diffqkv_pages_copy(ints(2), ints(2), cache(api), stream=STREAM, **heads))
        refused(api, lambda: api.diffqkv_pages_compact(cache(api), ints(6), stream=STREAM, **heads))
    made(api, lambda: api.diffqkv_pages_reserve(ints(3), cache(api), ints(6), 2, 4, stream=STREAM))
    made(api, lambda: api.diffqkv_pages_copy(ints(2), ints(2), cache(api, page_table=None), 2, 4, stream=STREAM))
    made(api, lambda: api.diffqkv_pages_compact(cache(api), ints(6), 2, 4, stream=STREAM))
    refused(api, lambda: api.diffqkv_pages_copy(ints(2), ints(2), cache(api), 2, 4, stream=STREAM,
                                                dst_cache=cache(api, k=z(6, 1, 16, 64))))


def test_the_pools_hold_what_the_cache_says(api):
    for kw in (dict(num_blocks=7), dict(page_size=32, max_seqlen=96), dict(k=z(6, 2, 64, 16).transpose(2, 3)),
               dict(page_table=ints(1, 3)), dict(page_table=None, page_size=0, max_seqlen=17)):
        refused(api, lambda: extend(api, c=cache(api, **kw)))
        refused(api, lambda: rope(api, c=cache(api, **kw)))
    made(api, lambda: extend(api, c=cache(api, num_blocks=5)))
    made(api, lambda: extend(api, c=cache(api, page_table=None, page_size=0, max_seqlen=16)))
    # pools of any shape with strides beside them: up to their last element, and not behind it
    flat = dict(k=z(6 * 16 * 2 * 64).view(-1, 64), v=z(6 * 16 * 4 * 64).view(-1, 64), k_strides=(2048, 64, 128),
                v_strides=(4096, 64, 256), num_blocks=6)
    made(api, lambda: extend(api, c=cache(api, **flat)))
    refused(api, lambda: extend(api, c=cache(api, **dict(flat, num_blocks=7))))
    refused(api, lambda: extend(api, c=cache(api, **dict(flat, k_strides=(2048, 64, 136)))))
    refused(api, lambda: extend(api, c=cache(api, **dict(flat, v=flat["v"][1:]))))


def test_the_status_word_is_an_int32(api):
    made(api, lambda: extend(api, dev_status=ints(1)))
    made(api, lambda: extend(api, dev_status=ints(4)[2:]))
    for bad in (z(1), torch.zeros(1, dtype=torch.uint8), ints(0)):
        refused(api, lambda: extend(api, dev_status=bad))
        refused(api, lambda: rope(api, dev_status=bad))
        refused(api, lambda: api.diffqkv_pages_free(ints(1), cache(api), ints(6), dev_status=bad, stream=STREAM))


def test_packed_structs_are_the_structures(api):
    """The bytes that the wrappers pack are what the ctypes structures hold."""
    cache_values = [16, 32, 1 << 40, -2, 3, 4, 5, 6, 48, 64, 7, 8, 9, 10]
    assert api._pack_cache(*cache_values) == bytes(api.CacheStruct(*cache_values))
    assert api._pack_shape(1, 2, 3, 4, 5, 6, 1, 0, 0.5) == bytes(api.ShapeStruct(1, 2, 3, 4, 5, 6, 1, 0, 0.5))
    assert api._pack_rope(16, 32, 64, 1, 1.5) == bytes(api.RopeStruct(16, 32, 64, 1, 1.5))
    assert api._pack_pages(16, 32, 48, 1, 2, 3, 4) == bytes(api.PagesStruct(16, 32, 48, 1, 2, 3, 4))


def test_pools_of_all_layers_heads(api):
    """Page calls take pools with the heads of every layer: the number of query heads that the shape needs is the least that
    both divide, since more than 65535 are refused."""
    for n_k, n_v, want in ((256, 256, 256), (128, 512, 512), (104, 416, 416), (2, 3, 6)):
        c = cache(api, k=z(2, n_k, 16, 8), v=z(2, n_v, 16, 8), page_table=ints(2, 3))
        for call in (lambda: api.diffqkv_pages_reserve(ints(3), c, ints(2), n_k, n_v, stream=STREAM),
                     lambda: api.diffqkv_pages_copy(ints(2), ints(2), c, n_k, n_v, stream=STREAM),
                     lambda: api.diffqkv_pages_compact(c, ints(2), n_k, n_v, stream=STREAM),
                     lambda: api.diffqkv_rope_append(None, z(5, n_k, 8), z(5, n_v, 8), ints(3), c, None, stream=STREAM)):
            shapes = [api.ShapeStruct.from_buffer_copy(a) for a in made(api, call)
                      if isinstance(a, bytes) and len(a) == C.sizeof(api.ShapeStruct)]
            assert (want, n_k, n_v) in [(s.n_q, s.n_k, s.n_v) for s in shapes]
            assert want <= 65535
