"""Calls without cu_new: one new token per sequence, which needs no bound on the new tokens."""
import dataclasses

import pytest
import torch

from paper_2509_10406_amd import binding as mb
from tests import packed_ref as ref
from tests.test_gpu_cache import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S,longest", [(1, 3000), (20, 700), (64, 1500), (70, 2500)])
def test_the_bound_is_known(S, longest, D, dtype):
    """The same bits with no bound, the right one and one that is too large, and for a call that gives the rows' offsets."""
    pairs = [(1 + (i * 617 + longest) % longest, 1) for i in range(S)]
    b = Batch(pairs, 8, 2, D, 32, dtype)
    want = None
    for max_new in (1, 0, S, 1 << 20):
        b.p = dataclasses.replace(b.p, max_new=max_new)
        before = [x.clone() for x in (b.cache.k, b.cache.v, b.cache.k_scale, b.cache.v_scale)]
        b.append(cu=None)
        got = (*b.attend(cu=None), b.cache.k.clone(), b.cache.v.clone(), b.cache.k_scale.clone(), b.cache.v_scale.clone())
        for x, y in zip((b.cache.k, b.cache.v, b.cache.k_scale, b.cache.v_scale), before):
            x.copy_(y)
        want = want or got
        assert all(torch.equal(x, y) for x, y in zip(got, want)), max_new
    b.p = dataclasses.replace(b.p, max_new=1)
    b.append()
    assert all(torch.equal(x, y) for x, y in zip(b.attend(), want))
    b.check_attend(want[:2])


def test_rows_of_many_sequences_without_a_bound():
    """As many sequences as a plan for pieces of prompts would have left without a workspace."""
    S = 2100
    b = Batch([(1 + 7 * i % 300, 1) for i in range(S)], 16, 8, 64, 64, torch.bfloat16)
    b.p = dataclasses.replace(b.p, max_new=0)
    b.append(cu=None)
    O, LSE = b.attend(cu=None)
    for i in (0, 1, 700, S - 1):   # each against the call for it alone
        one = dataclasses.replace(b.p, S=1, T=1)
        Oi, Li = mb.exact_attn_cache_fwd(one, b.Q[i:i + 1], None, b.lend[i:i + 1], b.table[i:i + 1], b.cache)
        want, tol = ref.cached(b.Q[i:i + 1], [0, 1], b.lens[i:i + 1], b.table[i:i + 1], *b.values(), 64, 64 ** -0.5)
        for o, l in ((O[i:i + 1], LSE[:, i:i + 1]), (Oi, Li)):
            ref.check("O", o, want["O"], tol["O"])
            ref.check("LSE", l, want["LSE"], tol["LSE"])
