"""What the Python forms of the ragged-batch calls refuse before the library is called (no GPU: the tensors lie on the host,
and a call that gets as far as the library is recorded, not made)."""
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
