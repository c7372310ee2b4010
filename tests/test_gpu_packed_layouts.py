"""Packed sequences, every kernel that a call may choose: strides, offsets past 32 bits, neighbours and padding that are not finite."""
import math

import pytest
import torch

from paper_2509_10406_amd import binding as mb
from tests import packed_ref as ref
from tests.test_gpu_packed import make, params

pytestmark = pytest.mark.gpu

NAMES = ("O", "LSE", "dQ", "dK", "dV")
FORMS = {  # lengths, heads, bound on the lengths (None: the longest, 0: none), type
    "short": ([90, 0, 150, 1, 33], 4, 2, None, torch.bfloat16),                 # tiles of 128 rows, dK / dV too at D = 64
    "short_heads_alone": ([333, 0, 600, 1, 64], 3, 3, None, torch.bfloat16),
    "between": ([1000, 0, 800, 1, 257], 4, 2, None, torch.bfloat16),            # some of both
    "long": ([1100, 0, 1600, 1, 257], 4, 2, 0, torch.bfloat16),                 # tiles of 256 rows
    "long_heads_alone": ([1100, 0, 1600, 1, 257], 3, 3, 0, torch.bfloat16),
    "fp32_few_tiles": ([333, 0, 150, 1, 64], 4, 2, None, torch.float32),
    "fp32_many_tiles": ([1100, 0, 1600, 1, 257], 16, 16, None, torch.float32),
}


def step(p, Q, K, V, dO, cud, out=None, grads=None):
    O, LSE = mb.exact_attn_packed_fwd(p, Q, K, V, cud, out=out)
    return (O, LSE, *mb.exact_attn_packed_bwd(p, Q, K, V, cud, O, LSE, dO, out=grads))


def case(form, D, **kw):
    lens, Hq, Hkv, max_len, dtype = FORMS[form]
    Q, K, V, dO, cu, cud = make(lens, Hq, Hkv, D, dtype, **kw)
    return Q, K, V, dO, cu, cud, params(lens, Q, K, max_len=max_len)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", list(FORMS))
def test_strides(form, D):
    Q, K, V, dO, cu, cud, p = case(form, D)
    want = step(p, Q, K, V, dO, cud)
    T, Hq, Hkv = p.T, p.Hq, p.Hkv
    heads_first = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    padded = lambda x: torch.nn.functional.pad(x, (0, 16))[..., :D]  # noqa: E731
    fused = torch.cat([Q, K, V, dO], 1)
    part = lambda a, n: fused[:, a:a + n]  # noqa: E731
    for q, k, v, g, lay in ((heads_first(Q), heads_first(K), heads_first(V), heads_first(dO), heads_first), (padded(Q), padded(K), padded(V), padded(dO), padded),
                            (part(0, Hq), part(Hq, Hkv), part(Hq + Hkv, Hkv), part(Hq + 2 * Hkv, Hq), heads_first)):
        got = step(p, q, k, v, g, cud, (lay(torch.zeros_like(Q)), torch.zeros_like(want[1])), tuple(lay(torch.zeros_like(x)) for x in (Q, K, V)))
        for n, a, b in zip(NAMES, got, want):
            assert torch.equal(a, b), n
    # a key and value of all rows, and a gradient, by strides of 0
    rep = [x[:1].expand(T, -1, D) for x in (K, V, dO)]
    for n, a, b in zip(NAMES, step(p, Q, *rep, cud), step(p, Q, *(x.contiguous() for x in rep), cud)):
        assert torch.equal(a, b), n


@pytest.mark.parametrize("order", ["rows", "heads"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", ["long", "short", "fp32_few_tiles", "fp32_many_tiles"])
def test_offsets_past_32_bits(form, D, order):
    """Views of one buffer whose last rows, or heads, lie more than 2^32 elements behind the first: the bits of the contiguous call."""
    _, Hq, Hkv, max_len, dtype = FORMS[form]
    lens = {"long": [1100, 0, 1600], "short": [150] * 17 + [83], "fp32_few_tiles": [1030, 40], "fp32_many_tiles": [1100, 0, 1600]}[form]
    Q, K, V, dO, cu, cud = make(lens, Hq, Hkv, D, dtype)
    p, T = params(lens, Q, K, max_len=max_len), Q.shape[0]
    want = step(p, Q, K, V, dO, cud)
    if order == "rows":   # all heads of all tensors side by side in wide rows
        token = (1 << 32) // (T - 30) // 8 * 8
        size, at = token * T, 0
    else:
        token, head = D, (1 << 32) // (Hq - 1) // 8 * 8 + 64
        size, at = head * (Hq - 1) + 16 * T * D, 0
    if size * Q.element_size() > torch.cuda.mem_get_info()[0] - (8 << 30):
        pytest.skip("needs more device memory")
    buf = torch.empty(size, dtype=dtype, device="cuda")
    views = []
    for x in (Q, K, V, dO, Q, Q, K, V):
        H = x.shape[1]
        stride, room = ((token, D, 1), H * D) if order == "rows" else ((token, head, 1), T * D)
        views.append(buf.as_strided((T, H, D), stride, at))
        at += room
    if order == "rows":
        assert at <= token and (T - 1) * token > 1 << 32
    for to, x in zip(views, (Q, K, V, dO)):
        to.copy_(x)
    q, k, v, g, o, *grads = views
    got = step(p, q, k, v, g, cud, (o, torch.zeros_like(want[1])), tuple(grads))
    for n, a, b in zip(NAMES, got, want):
        assert torch.equal(a, b), n


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", list(FORMS))
def test_a_sequence_keeps_its_numbers_to_itself(form, D, bad):
    Q, K, V, dO, cu, cud, p = case(form, D)
    clean = step(p, Q, K, V, dO, cud)
    for s in (0, 2):   # the sequence in front of the others, and the one between them
        x = [t.clone() for t in (Q, K, V, dO)]
        for t in x:
            t[cu[s]:cu[s + 1]] = bad
        for n, a, b in zip(NAMES, clean, step(p, *x, cud)):
            a, b = (a.t(), b.t()) if n == "LSE" else (a, b)
            for i in range(len(cu) - 1):
                assert i == s or torch.equal(a[cu[i]:cu[i + 1]], b[cu[i]:cu[i + 1]]), (n, i)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", list(FORMS))
def test_rows_of_no_sequence_are_left(form, D):
    Q, K, V, dO, cu, cud, p = case(form, D, before=37, behind=300)
    inside = torch.zeros(p.T, dtype=torch.bool, device="cuda")
    inside[cu[0]:cu[-1]] = True
    for x in (Q, K, V, dO):
        x[~inside] = math.nan
    mark = lambda t, *s: torch.full(s, 7.0, dtype=t, device="cuda")  # noqa: E731
    got = step(p, Q, K, V, dO, cud, (mark(Q.dtype, *Q.shape), mark(torch.float32, p.Hq, p.T)), tuple(mark(Q.dtype, *x.shape) for x in (Q, K, V)))
    want, tol = ref.packed(Q, K, V, cu, 1 / math.sqrt(D), dO, got[0], Q.dtype)
    for n, x in zip(NAMES, got):
        rows = x.t() if n == "LSE" else x
        assert (rows[~inside] == 7.0).all() and rows[inside].isfinite().all(), n
        ref.check(n, x, want[n], tol[n])
