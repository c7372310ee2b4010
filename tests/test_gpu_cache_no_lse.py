"""exact_attn_cache_fwd without LSE: the same O, in every kernel that writes one."""
import pytest
import torch

from paper_2509_10406_amd import binding as mb
from tests.test_gpu_cache import Batch

pytestmark = pytest.mark.gpu

PAIRS = {
    "whole": [(300, 1), (90, 1), (0, 0)],
    "divided": [(5000, 1), (700, 1)],
    "divided_among_many": [(60000, 1)],
    "divided_tiles_of_several": [(5000, 9), (700, 8)],
    "divided_pieces": [(5000, 200), (700, 90)],
    "pieces": [(200 + i, 100) for i in range(70)],
    "rows_without_keys": [(2, 5), (0, 3)],
}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("name", list(PAIRS))
def test_without_lse(name, D, dtype):
    b = Batch(PAIRS[name], 8, 2, D, 64, dtype)
    if name != "rows_without_keys":
        assert (mb.muse_cache_workspace_bytes(b.p) > 0) == name.startswith("divided")
    want = b.attend()
    O = torch.full_like(b.Q, 7.0)
    got = b.attend(out=(O, None))
    n = b.cu[-1]
    assert got[0] is O and got[1] is None and torch.equal(O[:n], want[0][:n]) and (O[n:] == 7.0).all()
