"""exact_attn_packed_fwd / exact_attn_packed_bwd against a 64-bit statement of the same attention."""
import math

import pytest
import torch

from paper_2509_10406_amd import binding as mb
from tests import packed_ref as ref

pytestmark = pytest.mark.gpu

LENS = {
    "one": [1],
    "empty_between": [0, 5, 0, 0, 2, 0],
    "tile_edges": [63, 64, 65, 1],
    "wide_edges": [255, 256, 257, 127, 128, 129],
    "ragged": [300, 1, 17, 0, 640, 33],
    "long": [1100, 40],
    "many": [(7 * i) % 23 for i in range(150)],
}
HEADS = [(2, 2), (6, 2), (5, 1)]


def make(lens, Hq, Hkv, D, dtype, seed=0, before=0, behind=0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T = before + sum(lens) + behind
    cu = [before + sum(lens[:i]) for i in range(len(lens) + 1)]
    x = [spread * torch.randn(T, h, D, generator=g, device="cuda") for h in (Hq, Hkv, Hkv, Hq)]
    Q, K, V, dO = (y.to(dtype) for y in x)
    return Q, K, V, dO, cu, torch.tensor(cu, dtype=torch.int32, device="cuda")


def params(lens, Q, K, grad=None, max_len=None, scale=0.0):
    dt = mb.BF16 if Q.dtype == torch.bfloat16 else mb.FP32
    return mb.PackedParams(S=len(lens), Hq=Q.shape[1], Hkv=K.shape[1], T=Q.shape[0], D=Q.shape[2],
                           max_len=max(lens) if max_len is None else max_len, dtype=dt, grad_dtype=dt if grad is None else grad, scale=scale)


def run_and_check(p, Q, K, V, dO, cu, cud, what=""):
    O, LSE = mb.exact_attn_packed_fwd(p, Q, K, V, cud)
    grads = mb.exact_attn_packed_bwd(p, Q, K, V, cud, O, LSE, dO)
    scale = p.scale or 1 / math.sqrt(p.D)
    want, tol = ref.packed(Q, K, V, cu, scale, dO, O, p.torch_grad_dtype)
    for n, x in zip(("O", "LSE", "dQ", "dK", "dV"), (O, LSE, *grads)):
        ref.check(f"{what} {n}", x, want[n], tol[n])
    return (O, LSE, *grads)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", HEADS)
@pytest.mark.parametrize("name", list(LENS))
def test_against_64_bits(name, Hq, Hkv, D, dtype):
    lens = LENS[name]
    Q, K, V, dO, cu, cud = make(lens, Hq, Hkv, D, dtype)
    run_and_check(params(lens, Q, K), Q, K, V, dO, cu, cud, name)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [[1500, 700, 90], [2600]])
def test_long_sequences(lens, D):
    """Enough tiles for every kernel of long sequences, grouped heads."""
    Q, K, V, dO, cu, cud = make(lens, 16, 4, D, torch.bfloat16)
    run_and_check(params(lens, Q, K), Q, K, V, dO, cu, cud)


@pytest.mark.parametrize("grad", [mb.BF16, mb.FP32])
@pytest.mark.parametrize("Hq,Hkv,lens", [(3, 3, [640, 0, 513, 129, 1]), (12, 4, [192, 1, 127, 0, 65, 129])])
def test_short_sequences(Hq, Hkv, lens, grad):
    """The kernels of 128 rows, with and without grouped heads."""
    Q, K, V, dO, cu, cud = make(lens, Hq, Hkv, 64, torch.bfloat16)
    run_and_check(params(lens, Q, K, grad=grad), Q, K, V, dO, cu, cud)


@pytest.mark.parametrize("D", [64, 128])
def test_many_tiles_in_fp32(D):
    """More tiles than the form for few of them takes."""
    lens = [700, 650, 0, 720, 690, 1, 640, 660]
    Q, K, V, dO, cu, cud = make(lens, 16, 16, D, torch.float32)
    run_and_check(params(lens, Q, K), Q, K, V, dO, cu, cud)


@pytest.mark.parametrize("D", [64, 128])
def test_fp32_gradients_of_bf16_inputs_and_a_scale(D):
    lens = [130, 3, 400]
    Q, K, V, dO, cu, cud = make(lens, 4, 2, D, torch.bfloat16)
    run_and_check(params(lens, Q, K, grad=mb.FP32, scale=0.31), Q, K, V, dO, cu, cud)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_scores(dtype):
    """Peaked rows: the running maximum moves far and often."""
    lens = [500, 77]
    Q, K, V, dO, cu, cud = make(lens, 2, 1, 64, dtype, spread=4.0)
    run_and_check(params(lens, Q, K), Q, K, V, dO, cu, cud)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("max_len", [0, 1, 100000])
def test_the_bound_on_lengths_is_a_hint(max_len, dtype):
    lens = [400, 3, 90]
    Q, K, V, dO, cu, cud = make(lens, 4, 2, 64, dtype)
    run_and_check(params(lens, Q, K, max_len=max_len), Q, K, V, dO, cu, cud)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", HEADS)
@pytest.mark.parametrize("name", list(LENS))
def test_without_a_bound(name, Hq, Hkv, D):
    """No bound on the lengths: the kernels of long sequences, whatever the lengths are."""
    lens = LENS[name] + [0, 0]
    Q, K, V, dO, cu, cud = make(lens, Hq, Hkv, D, torch.bfloat16, behind=2700)   # with their rows, T is past every line
    run_and_check(params(lens, Q, K, max_len=0), Q, K, V, dO, cu, cud, name)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_of_no_sequence_are_left(D, dtype):
    """Rows in front of the first and behind the last sequence: never read as numbers, never written."""
    lens = [70, 0, 300]
    Q, K, V, dO, cu, cud = make(lens, 4, 2, D, dtype, before=37, behind=300)
    inside = torch.zeros(Q.shape[0], dtype=torch.bool, device="cuda")
    inside[cu[0]:cu[-1]] = True
    for x in (Q, K, V, dO):
        x[~inside] = math.nan
    p = params(lens, Q, K)
    mark = lambda t, *s: torch.full(s, 7.0, dtype=t, device="cuda")  # noqa: E731
    O, LSE = mark(dtype, *Q.shape), mark(torch.float32, 4, Q.shape[0])
    mb.exact_attn_packed_fwd(p, Q, K, V, cud, out=(O, LSE))
    grads = tuple(mark(dtype, *x.shape) for x in (Q, K, V))
    mb.exact_attn_packed_bwd(p, Q, K, V, cud, O, LSE, dO, out=grads)
    for x in (O, LSE.t(), *grads):
        assert (x[~inside] == 7.0).all() and x[inside].isfinite().all()
    want, tol = ref.packed(Q, K, V, cu, 1 / math.sqrt(D), dO, O, dtype)
    for n, x in zip(("O", "LSE", "dQ", "dK", "dV"), (O, LSE, *grads)):
        ref.check(n, x, want[n], tol[n])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_sequence_keeps_its_numbers_to_itself(bad, D, dtype):
    """Rows that are not finite in one sequence: its neighbours, in the same tiles of memory, get the same bits."""
    lens = [100, 60, 320]
    Q, K, V, dO, cu, cud = make(lens, 4, 2, D, dtype)
    p = params(lens, Q, K)

    def results():
        O, LSE = mb.exact_attn_packed_fwd(p, Q, K, V, cud)
        return (O, LSE.t(), *mb.exact_attn_packed_bwd(p, Q, K, V, cud, O, LSE, dO))

    clean = results()
    for x in (Q, K, V, dO):
        x[cu[1]:cu[2]] = bad
    for a, b in zip(clean, results()):
        for s in (0, 2):
            assert torch.equal(a[cu[s]:cu[s + 1]], b[cu[s]:cu[s + 1]])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
def test_strides(D, dtype):
    """Heads first, slices of a fused projection, padded rows, repeated heads; outputs with strides of their own."""
    lens, Hq, Hkv = [90, 0, 333, 1], 4, 2
    Q, K, V, dO, cu, cud = make(lens, Hq, Hkv, D, dtype)
    T, p = Q.shape[0], params(lens, Q, K)
    O, LSE = mb.exact_attn_packed_fwd(p, Q, K, V, cud)
    want = (O, LSE, *mb.exact_attn_packed_bwd(p, Q, K, V, cud, O, LSE, dO))
    heads_first = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    fused = torch.cat([Q, K, V], 1)
    padded = lambda x: torch.nn.functional.pad(x, (0, 16))[..., :D]  # noqa: E731
    for q, k, v, g, make_out in ((heads_first(Q), heads_first(K), heads_first(V), heads_first(dO), heads_first),
                                 (fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:], padded(dO), padded)):
        out = (make_out(torch.zeros_like(Q)), torch.zeros_like(LSE))
        mb.exact_attn_packed_fwd(p, q, k, v, cud, out=out)
        grads = tuple(make_out(torch.zeros_like(x)) for x in (Q, K, V))
        mb.exact_attn_packed_bwd(p, q, k, v, cud, *out, g, out=grads)
        for a, b in zip(want, (*out, *grads)):
            assert torch.equal(a, b)
    fused_grads = torch.zeros_like(fused)
    mb.exact_attn_packed_bwd(p, Q, K, V, cud, O, LSE, dO, out=(fused_grads[:, :Hq], fused_grads[:, Hq:Hq + Hkv], fused_grads[:, Hq + Hkv:]))
    assert torch.equal(fused_grads, torch.cat(want[2:], 1))
    # one key and value head for all, repeated by a stride of 0, is the grouped call
    k1, v1 = K[:, :1], V[:, :1]
    a = mb.exact_attn_packed_fwd(mb.PackedParams(S=4, Hq=Hq, Hkv=1, T=T, D=D, dtype=p.dtype), Q, k1, v1, cud)
    b = mb.exact_attn_packed_fwd(mb.PackedParams(S=4, Hq=Hq, Hkv=Hq, T=T, D=D, dtype=p.dtype), Q, k1.expand(T, Hq, D), v1.expand(T, Hq, D), cud)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
def test_equal_lengths_are_the_batched_call(D, dtype):
    """Against exact_attn_fwd / exact_attn_bwd over a batch of the same sequences: both are within their bounds of the 64-bit result, so
    within two of each other."""
    B, N, Hq, Hkv = 3, 384, 4, 2
    lens = [N] * B
    Q, K, V, dO, cu, cud = make(lens, Hq, Hkv, D, dtype)
    p = params(lens, Q, K)
    O, LSE = mb.exact_attn_packed_fwd(p, Q, K, V, cud)
    packed = (O, LSE, *mb.exact_attn_packed_bwd(p, Q, K, V, cud, O, LSE, dO))
    b = mb.Params(B=B, Hq=Hq, Hkv=Hkv, N=N, D=D, dtype=p.dtype, grad_dtype=p.grad_dtype)
    apart = lambda x: x.view(B, N, -1, D).transpose(1, 2).contiguous()  # noqa: E731
    Ob, Lb = mb.exact_attn_fwd(b, apart(Q), apart(K), apart(V))
    grads = mb.exact_attn_bwd(b, apart(Q), apart(K), apart(V), Ob, Lb, apart(dO))
    _, tol = ref.packed(Q, K, V, cu, 1 / math.sqrt(D), dO, O, dtype)
    back = lambda x: x.transpose(1, 2).reshape(B * N, -1, D)  # noqa: E731
    for n, x, y in zip(("O", "dQ", "dK", "dV"), (packed[0], *packed[2:]), (Ob, *grads)):
        ref.check(n, x, back(y).double(), 2 * tol[n])
    # its normaliser adds up the weights as rounded to bf16
    assert (LSE.view(Hq, B, N).transpose(0, 1) - Lb).abs().max() <= (2.0 ** -8 if dtype == torch.bfloat16 else 1e-5)


def test_the_same_bits_every_time():
    lens = [900, 5, 300, 0, 64]
    Q, K, V, dO, cu, cud = make(lens, 8, 2, 128, torch.bfloat16)
    p = params(lens, Q, K)
    first = None
    for _ in range(3):
        O, LSE = mb.exact_attn_packed_fwd(p, Q, K, V, cud)
        got = (O, LSE, *mb.exact_attn_packed_bwd(p, Q, K, V, cud, O, LSE, dO))
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_captured_into_graphs(dtype):
    """Two graphs of a forward and backward, replayed in turn with new inputs and eager calls in between."""
    cases = []
    for lens, seed in (([300, 20], 1), ([64, 0, 500], 2)):
        Q, K, V, dO, cu, cud = make(lens, 4, 2, 64, dtype, seed=seed)
        p = params(lens, Q, K)

        def step(p=p, Q=Q, K=K, V=V, dO=dO, cud=cud):
            O, LSE = mb.exact_attn_packed_fwd(p, Q, K, V, cud)
            return (O, LSE, *mb.exact_attn_packed_bwd(p, Q, K, V, cud, O, LSE, dO))

        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        cases.append((graph, out, step, (Q, K, V, dO)))
    for turn in range(3):
        for graph, out, step, inputs in cases:
            for x in inputs:
                x.mul_(0.75).add_(0.01 * turn)
            graph.replay()
            want = step()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_on_another_stream():
    lens = [500, 44]
    Q, K, V, dO, cu, cud = make(lens, 4, 2, 64, torch.bfloat16)
    p = params(lens, Q, K)
    O, LSE = mb.exact_attn_packed_fwd(p, Q, K, V, cud)
    want = mb.exact_attn_packed_bwd(p, Q, K, V, cud, O, LSE, dO)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for st in streams:   # both at once
        with torch.cuda.stream(st):
            o, l = mb.exact_attn_packed_fwd(p, Q, K, V, cud)
            got.append((o, l, *mb.exact_attn_packed_bwd(p, Q, K, V, cud, o, l, dO)))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip((O, LSE, *want), g))


def test_gradients_against_differences():
    """<gradient, u> against central differences of sum(O dO) in 64 bits along u, extrapolated; what the extrapolation is off by is
    less than the change that it makes."""
    lens, D = [40, 1, 75], 64
    Q, K, V, dO, cu, cud = make(lens, 4, 2, D, torch.float32)
    p = params(lens, Q, K)
    O, LSE = mb.exact_attn_packed_fwd(p, Q, K, V, cud)
    grads = mb.exact_attn_packed_bwd(p, Q, K, V, cud, O, LSE, dO)
    _, tol = ref.packed(Q, K, V, cu, 1 / math.sqrt(D), dO, O, torch.float32)
    g = torch.Generator(device="cuda").manual_seed(3)
    inputs = [x.double() for x in (Q, K, V)]
    for i, name in enumerate(("dQ", "dK", "dV")):
        u = torch.randn(inputs[i].shape, generator=g, device="cuda", dtype=torch.float64)

        def value(t):
            x = list(inputs)
            x[i] = x[i] + t * u
            return float((ref.packed(*x, cu, 1 / math.sqrt(D))[0]["O"] * dO.double()).sum())

        diff = lambda t: (value(t) - value(-t)) / (2 * t)  # noqa: E731
        a, b = diff(2.0 ** -7), diff(2.0 ** -8)
        got = float((grads[i].double() * u).sum())
        assert abs(got - (4 * b - a) / 3) <= abs(a - b) + float((tol[name] * u.abs()).sum()), name
