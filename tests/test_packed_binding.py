"""CPU-only: what the binding of packed sequences and of the paged cache hands to the library, on tensors that are taken for device
tensors, and limits that are checked on the host; nothing is launched."""
import ctypes as C

import pytest
import torch

from paper_2509_10406_amd import binding as mb

P = dict(S=2, Hq=4, Hkv=2, T=2, D=64, pages=5, page=16, table_cols=3, max_new=1)


@pytest.fixture
def cache(monkeypatch):
    monkeypatch.setattr(mb, "_on_gpu", lambda t: t.device)
    return mb.kv_cache(mb.CacheParams(**P), device="cpu")


def addresses(cache):
    p = mb.CacheParams(**P)
    return mb._cache_ptrs(p, None, torch.zeros(2, dtype=torch.int32), torch.zeros(2, 3, dtype=torch.int32), cache, torch.device("cpu"))[1]


@pytest.mark.parametrize("name", ["k", "v", "k_scale", "v_scale"])
def test_replaced_cache_tensors(cache, name):
    """A cache that was moved out and back has other addresses; tensors that do not fit any more are refused."""
    at = ["k", "v", "k_scale", "v_scale"].index(name)
    t = getattr(cache, name)
    before = addresses(cache)
    kept = t.data              # so that the new tensor lies elsewhere
    t.data = kept.clone()
    assert t.data_ptr() != kept.data_ptr()
    after = addresses(cache)
    assert after[at] == t.data_ptr() and all(a == b for i, (a, b) in enumerate(zip(after, before)) if i != at)
    for bad in (kept[:1], kept.transpose(0, 1), kept.to(torch.float64), kept[..., None]):
        t.data = bad
        with pytest.raises(mb.MuseError, match=f"cache.{name}"):
            addresses(cache)
    t.data = kept
    assert addresses(cache) == before


def test_a_cache_that_does_not_fit_the_params(cache):
    for kw in (dict(pages=6), dict(page=32), dict(Hkv=4), dict(D=128)):
        p = mb.CacheParams(**(P | kw))
        with pytest.raises(mb.MuseError, match="cache"):
            mb._cache_ptrs(p, None, torch.zeros(2, dtype=torch.int32), torch.zeros(2, 3, dtype=torch.int32), cache, torch.device("cpu"))
    with pytest.raises(mb.MuseError, match="cache.v"):
        mb.KVCache(cache.k, cache.k, cache.k_scale, cache.v_scale)


@pytest.mark.parametrize("page", [16, 128])
def test_positions_and_the_units_behind_them_are_31_bits(page):
    """Attention goes by units of 256 keys and asks for the table's entries up to two units ahead: positions end that far below 2^31."""
    most = (2**31 - 1024) // page
    for cols, rc in ((most, 0), (most + 1, -2), ((2**31 - 1) // page, -2)):
        got = C.c_size_t(0)
        p = mb.CacheParams(**(P | dict(page=page, table_cols=cols)))
        assert mb.load().muse_cache_workspace_bytes(C.byref(p._c), C.byref(got)) == rc, cols


@pytest.mark.parametrize("S,dtype", [(64, mb.BF16), (4096, mb.BF16), (4096, mb.FP32), (2, mb.FP32)])
def test_workspace_of_single_tokens_without_a_bound(S, dtype):
    """A call without cu_new has one new token per sequence, also where the params hold no bound: the workspace is enough for that plan."""
    size = lambda n: mb.muse_cache_workspace_bytes(mb.CacheParams(S=S, Hq=32, Hkv=8, T=S, D=128, pages=9, page=64, table_cols=200,  # noqa: E731
                                                                  max_new=n, dtype=dtype))
    assert size(0) >= size(1) > 0


def test_tensors_on_another_device_than_the_current_one(monkeypatch):
    """The call is made on the tensors' device, on that device's current stream."""
    now, calls = [0], []

    class device:
        def __init__(self, d):
            self.to = d.index

        def __enter__(self):
            self.was, now[0] = now[0], self.to

        def __exit__(self, *_):
            now[0] = self.was

    class library:
        @staticmethod
        def exact_attn_packed_fwd(p, *args):
            calls.append((now[0], args))
            return 0

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: now[0], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 100 + i, raising=False)
    monkeypatch.setattr(mb, "load", lambda: library)
    for index in (0, 1):
        mb._packed_call("exact_attn_packed_fwd", torch.device("cuda", index), mb._PackedParams(), 5)
    assert calls == [(0, (5, 100)), (1, (5, 101))] and now == [0]
