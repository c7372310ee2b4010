"""CPU-only: what the entry points of packed sequences and of the paged cache refuse, before anything is launched; and the 64-bit
statements that the GPU tests compare with, against plain sums."""
import ctypes as C
import dataclasses
import math

import pytest
import torch

from paper_2509_10406_amd import binding as mb
from tests import packed_ref as ref

FAKE = 4096  # an aligned address; never dereferenced: every call here fails a check on the host


def packed(**kw):
    p = mb.PackedParams(**(dict(S=3, Hq=8, Hkv=2, T=100, D=64, grad_dtype=mb.BF16) | kw))
    pc = mb._PackedParams.from_buffer_copy(p._c)
    for n in ("q", "o", "dout", "dq"):
        getattr(pc, n).token, getattr(pc, n).head = p.Hq * p.D, p.D
    for n in ("k", "v", "dk", "dv"):
        getattr(pc, n).token, getattr(pc, n).head = p.Hkv * p.D, p.D
    return pc


def cache(**kw):
    p = mb.CacheParams(**(dict(S=3, Hq=8, Hkv=2, T=7, D=64, pages=10, page=32, table_cols=4) | kw))
    pc = mb._CacheParams.from_buffer_copy(p._c)
    pc.q.token, pc.q.head = p.Hq * p.D, p.D
    pc.o.token, pc.o.head = p.Hq * p.D, p.D
    pc.k.token, pc.k.head = p.Hkv * p.D, p.D
    pc.v.token, pc.v.head = p.Hkv * p.D, p.D
    return pc


def fwd(pc, args=(FAKE,) * 6, ws=FAKE, size=1 << 40):
    return mb.load().exact_attn_packed_fwd(C.byref(pc), *args, ws, size, 0)


def bwd(pc, args=(FAKE,) * 10, ws=FAKE, size=1 << 40):
    return mb.load().exact_attn_packed_bwd(C.byref(pc), *args, ws, size, 0)


def append(pc, args=(FAKE,) * 9):
    return mb.load().exact_attn_cache_append(C.byref(pc), *args, 0)


def attend(pc, args=(FAKE,) * 10, ws=FAKE, size=1 << 40):
    return mb.load().exact_attn_cache_fwd(C.byref(pc), *args, ws, size, 0)


INVALID, UNSUPPORTED, SMALL = -1, -2, -3
COMMON = [(dict(S=0), INVALID), (dict(Hq=0), INVALID), (dict(Hkv=3), INVALID), (dict(T=0), INVALID), (dict(dtype=2), INVALID),
          (dict(scale=-1.0), INVALID), (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID), (dict(D=80), UNSUPPORTED),
          (dict(T=(1 << 27) + 1), UNSUPPORTED), (dict(Hq=8192), UNSUPPORTED)]


@pytest.mark.parametrize("kw,rc", COMMON + [(dict(max_len=-1), INVALID), (dict(S=1 << 20), UNSUPPORTED), (dict(T=1 << 26), UNSUPPORTED), (dict(grad_dtype=2), INVALID), (dict(dtype=mb.FP32), INVALID)])
def test_packed_params(kw, rc):
    assert fwd(packed(**kw)) == rc and bwd(packed(**kw)) == rc


@pytest.mark.parametrize("kw,rc", COMMON + [(dict(pages=0), INVALID), (dict(table_cols=0), INVALID), (dict(max_new=-1), INVALID),
                                            (dict(page=48), UNSUPPORTED), (dict(page=8), UNSUPPORTED),
                                            (dict(table_cols=1 << 27), UNSUPPORTED), (dict(S=1 << 20, table_cols=1 << 24), UNSUPPORTED),
                                            (dict(T=1 << 27, Hq=32), UNSUPPORTED)])
def test_cache_params(kw, rc):
    assert append(cache(**kw)) == rc and attend(cache(**kw)) == rc
    got = C.c_size_t(0)
    assert mb.load().muse_cache_workspace_bytes(C.byref(cache(**kw)), C.byref(got)) == rc


def test_null_pointers_alignment_and_workspaces():
    assert mb.load().exact_attn_packed_fwd(0, *(FAKE,) * 7, 1 << 40, 0) == INVALID
    for call, n, may_be_null in ((fwd, 6, ()), (bwd, 10, ()), (append, 9, ()), (attend, 10, (9,))):
        pc = packed() if n in (6,) or call is bwd else cache()
        for i in range(n):
            if i not in may_be_null:
                args = [FAKE] * n
                args[i] = 0
                assert call(pc, tuple(args)) == INVALID, (call, i)   # cu_new NULL: T is not S here
    for call, pc, n, rows in ((fwd, packed(), 6, (0, 1, 2, 4)), (bwd, packed(), 10, (0, 1, 2, 4, 6, 7, 8, 9)), (append, cache(), 9, (0, 1, 5, 6)),
                              (attend, cache(), 10, (0, 4, 5, 8))):
        for i in rows:
            args = [FAKE] * n
            args[i] += 8
            assert call(pc, tuple(args)) == INVALID, (call, i)
    assert bwd(packed(), size=64) == SMALL and bwd(packed(), ws=0) == INVALID and bwd(packed(), ws=FAKE + 16) == INVALID


def test_strides():
    for n, call in (("q", fwd), ("k", fwd), ("v", fwd), ("o", fwd), ("dout", bwd), ("dq", bwd), ("dk", bwd), ("dv", bwd)):
        for token, head, rc in ((-64, 64, INVALID), (516, 64, INVALID), (512, 68, INVALID), ((1 << 22) + 64, 64, UNSUPPORTED),
                                (512, 1 << 41, UNSUPPORTED)):
            pc = packed()
            getattr(pc, n).token, getattr(pc, n).head = token, head
            assert call(pc) == rc, (n, token, head)
    for n, call in (("o", fwd), ("dq", bwd), ("dk", bwd)):   # rows of an output that meet
        for token, head in ((0, 64), (64, 64), (512, 0), (448, 64) if n != "dk" else (64, 64), (64, 64 * 99)):
            pc = packed()
            getattr(pc, n).token, getattr(pc, n).head = token, head
            assert call(pc) == INVALID, (n, token, head)
    pc = packed()
    pc.o.token, pc.o.head = 64, 6400      # heads first: fine, so the next check speaks
    assert fwd(pc, (FAKE, FAKE, FAKE, 0, FAKE, FAKE)) == INVALID
    pc = cache()
    pc.o.token = 0
    assert attend(pc) == INVALID


def test_binding_refuses_what_does_not_fit():
    p = mb.PackedParams(S=1, Hq=2, Hkv=1, T=4, D=64)
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(mb.MuseError, match="device-resident"):
        mb.exact_attn_packed_fwd(p, x, x, x, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(dataclasses.FrozenInstanceError):
        p.T = 5
    rows, cpu = mb._Rows(), torch.device("cpu")
    assert mb._packed_rows(rows, x, "Q", 4, 2, 64, torch.bfloat16, cpu) == x.data_ptr() and (rows.token, rows.head) == (128, 64)
    for bad in (x.float(), x[:3], x.transpose(1, 2), torch.zeros(4, 2, 128, dtype=torch.bfloat16)[..., ::2]):
        with pytest.raises(mb.MuseError, match="Q"):
            mb._packed_rows(rows, bad, "Q", 4, 2, 64, torch.bfloat16, cpu)
    cu = torch.zeros(4, dtype=torch.int32)
    for bad in (cu.long(), cu[:3], torch.zeros(8, dtype=torch.int32)[::2]):
        with pytest.raises(mb.MuseError, match="cu"):
            mb._whole(bad, "cu", (4,), torch.int32, cpu)
    with pytest.raises(mb.MuseError, match="unsupported"):
        mb.muse_cache_workspace_bytes(mb.CacheParams(S=1, Hq=1, Hkv=1, T=1, D=64, pages=1, page=20, table_cols=1))
    assert mb.muse_packed_workspace_bytes(p, mb.WS_EXACT_BWD) >= 4 * 2 * 4


def test_reference_attention_is_the_softmax():
    g = torch.Generator().manual_seed(0)
    q, k, v, dO = (torch.randn(7, 5, generator=g, dtype=torch.float64, requires_grad=i < 3) for i in range(4))
    z = (q @ k.T * 0.3).masked_fill(torch.triu(torch.ones(7, 7, dtype=torch.bool), 1), -math.inf)
    o = torch.softmax(z, 1) @ v
    o.backward(dO)
    got, _ = ref.head(q.detach(), k.detach(), v.detach(), 0, 0.3, dO)
    assert torch.allclose(got["O"], o.detach()) and torch.allclose(got["LSE"], torch.logsumexp(z, 1).detach())
    assert torch.allclose(got["dQ"], q.grad) and torch.allclose(got["dK"], k.grad) and torch.allclose(got["dV"], v.grad)


def test_reference_rounding_is_the_type():
    x = torch.cat([torch.linspace(-448, 448, 40001), torch.linspace(-0.02, 0.02, 4001), torch.tensor([0.0, 2.0 ** -10, 3 * 2.0 ** -10, 448.0])])
    assert torch.equal(ref.e4m3(x.double()), x.to(torch.float8_e4m3fn).double())
    for amax, want in ((448.0, 1.0), (448.5, 2.0), (224.0, 0.5), (1e-9, 2.0 ** -38), (0.0, 2.0 ** -100)):
        assert ref.least_scale(amax) == want
