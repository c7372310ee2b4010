"""The entry points of packed sequences and of the paged cache on a workspace that holds a kept forward state: what they write there
is not taken for that state afterwards."""
import dataclasses

import pytest
import torch

from paper_2509_10406_amd import binding as mb
from tests.test_gpu_cache import Batch
from tests.test_gpu_muse import CASES, dev, generate, oracle_clustering, small
from tests.test_gpu_packed import make, params

STAMP = 32   # bytes at the head


def test_scratch_lies_behind_the_stamp():
    p = mb.PackedParams(S=1, Hq=2, Hkv=1, T=100, D=64)
    assert mb.muse_packed_workspace_bytes(p, mb.WS_EXACT_BWD) >= 256 + 4 * 2 * 100


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_packed_backward_clears_it(dtype):
    """Rows of no sequence in front, for which nothing is written to the scratch."""
    lens = [40, 3]
    Q, K, V, dO, cu, cud = make(lens, 2, 1, 64, dtype, before=70, behind=5)
    p = params(lens, Q, K)
    O, LSE = mb.exact_attn_packed_fwd(p, Q, K, V, cud)
    want = mb.exact_attn_packed_bwd(p, Q, K, V, cud, O, LSE, dO)
    ws = torch.full((mb.muse_packed_workspace_bytes(p, mb.WS_EXACT_BWD),), 7, dtype=torch.uint8, device="cuda")
    got = mb.exact_attn_packed_bwd(p, Q, K, V, cud, O, LSE, dO, ws=ws)
    assert (ws[:STAMP] == 0).all()
    assert all(torch.equal(a[cu[0]:cu[-1]], b[cu[0]:cu[-1]]) for a, b in zip(want, got))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,new", [(torch.bfloat16, 1), (torch.bfloat16, 9), (torch.bfloat16, 200), (torch.float32, 1)])
def test_cache_attention_clears_it(dtype, new):
    b = Batch([(6000, new), (2000, new)], 8, 2, 64, 64, dtype)
    want = b.attend()
    size = mb.muse_cache_workspace_bytes(b.p)
    assert size > 256   # the contexts are divided
    ws = torch.full((size,), 7, dtype=torch.uint8, device="cuda")
    got = b.attend(ws=ws)
    assert (ws[:STAMP] == 0).all() and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.gpu
@pytest.mark.parametrize("by", ["packed", "cache"])
def test_a_kept_state_that_was_written_to_is_refused(by):
    base, kw = CASES["cfg2_small"]
    w = small(base, **kw)
    d, p = generate(w, need_dO=True), mb.params_for(w)
    pk = dataclasses.replace(p, flags=mb.FLAG_KEEP_FWD_STATE)
    qc, aq, ak = oracle_clustering(w, d, p)
    Q, K, V, dO = (dev(d[x], p) for x in ("Q", "K", "V", "dO"))
    cl = (torch.tensor(qc).cuda(), torch.tensor(aq).cuda(), torch.tensor(ak).cuda())
    ws = torch.zeros(mb.muse_workspace_bytes(pk, mb.WS_BWD)[1], dtype=torch.uint8, device="cuda")
    O, LSE, selc, selb = mb.muse_fwd(pk, Q, K, V, *cl, ws=ws)
    lens = [40, 3]
    q, k, v, g, cu, cud = make(lens, 2, 1, 64, torch.bfloat16, before=70)
    pp = params(lens, q, k)
    o, lse = mb.exact_attn_packed_fwd(pp, q, k, v, cud, ws=ws)   # needs no workspace: the state is still there
    mb.muse_bwd(pk, Q, K, V, O, LSE, dO, *cl, selc, selb, ws=ws)
    if by == "packed":
        mb.exact_attn_packed_bwd(pp, q, k, v, cud, o, lse, g, ws=ws)
    else:
        b = Batch([(6000, 1)], 2, 1, 64, 64, torch.bfloat16)
        assert 256 < mb.muse_cache_workspace_bytes(b.p) <= ws.numel()
        b.attend(ws=ws)
    with pytest.raises(mb.MuseError, match="forward state"):
        mb.muse_bwd(pk, Q, K, V, O, LSE, dO, *cl, selc, selb, ws=ws)
