"""How far a row that is not finite reaches inside its own sequence (its neighbours: test_gpu_packed_layouts.py): to what attends to it, and
beyond that no further than include/muse.h says."""
import math

import pytest
import torch

from paper_2509_10406_amd import binding as mb
from tests.test_gpu_cache import Batch
from tests.test_gpu_packed_layouts import FORMS, case, step

pytestmark = pytest.mark.gpu

PACKED_REACH, CACHE_REACH = 255, 94


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", list(FORMS))
def test_packed(form, D, bad):
    Q, K, V, dO, cu, cud, p = case(form, D)
    O, LSE, dQ, dK, dV = step(p, Q, K, V, dO, cud)
    beg, end = cu[2], cu[3]
    j = beg + (end - beg) * 3 // 5
    same = lambda a, b, lo, hi: torch.equal(a[lo:max(lo, hi)], b[lo:max(lo, hi)])  # noqa: E731
    for name, x in (("Q", Q), ("K", K), ("V", V), ("dO", dO)):
        kept = x[j].clone()
        x[j] = bad
        o, lse, dq, dk, dv = step(p, Q, K, V, dO, cud)
        x[j] = kept
        # rows in front, further than the reach: what they attend to is as it was
        for a, b in ((o, O), (lse.t(), LSE.t()), (dq, dQ)):
            assert same(a, b, 0, j - PACKED_REACH), name
        if name == "V":
            assert torch.equal(lse, LSE)
        if name in ("Q", "dO"):   # keys behind the row, and other queries
            for a, b in ((dk, dK), (dv, dV)):
                assert same(a, b, j + PACKED_REACH + 1, p.T), name
            for a, b in ((o, O), (dq, dQ)):
                assert same(a, b, j + PACKED_REACH + 1, p.T), name
        assert not (o[j].isfinite() if name != "dO" else dq[j].isfinite()).any(), name
        for a, b in zip((o, lse.t(), dq, dk, dv), (O, LSE.t(), dQ, dK, dV)):   # the other sequences
            assert same(a, b, 0, beg) and same(a, b, end, p.T), name


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,new", [(2, 2, 300), (2, 2, 50), (4, 1, 3), (4, 2, 100)])
def test_cache(Hq, Hkv, new, D, dtype):
    b = Batch([(200, 1), (900, new), (70, min(new, 70))], Hq, Hkv, D, 32, dtype)
    O, LSE = b.attend()
    L, first, beg, end = 900, 900 - new, b.cu[1], b.cu[2]
    for pos in (L - 1, first + new // 2, first, 100):
        pid, at = int(b.table[1, pos // 32]), pos % 32
        row = beg + max(pos - first, 0)        # the first query that attends to it
        for keys, cache in ((True, b.cache.k[pid, :, at]), (False, b.cache.v[pid, :, :, at])):
            kept = cache.clone()
            cache.fill_(127)
            o, lse = b.attend()
            cache.copy_(kept)
            clear = row if keys else max(row - CACHE_REACH, beg)
            for lo, hi in ((0, beg), (beg, clear), (end, b.p.T)):
                assert torch.equal(o[lo:hi], O[lo:hi]), (keys, pos, lo, hi)
            assert not o[row:end].isfinite().any(), (keys, pos)
            if keys:
                assert torch.equal(lse[:, :row], LSE[:, :row]) and torch.equal(lse[:, end:], LSE[:, end:]) and lse[:, row:end].isnan().all(), pos
            else:
                assert torch.equal(lse, LSE), pos
