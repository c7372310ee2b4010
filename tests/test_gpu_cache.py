"""exact_attn_cache_append and exact_attn_cache_fwd against 64-bit statements: stored bytes exactly, attention within its rounding."""
import math

import pytest
import torch

from paper_2509_10406_amd import binding as mb
from tests import packed_ref as ref

pytestmark = pytest.mark.gpu

BATCHES = {  # (length, new tokens) of every sequence
    "single": [(1, 1)],
    "tokens": [(1, 1), (2, 1), (16, 1), (17, 1), (64, 1), (65, 1), (200, 1), (129, 1)],
    "prompts": [(1, 1), (16, 16), (17, 17), (70, 70), (130, 130)],
    "pieces": [(90, 31), (33, 33), (300, 2), (64, 0), (0, 0), (129, 65), (257, 130)],
    "long": [(1500, 1), (3, 3), (2600, 5)],
    "drafts": [(700, 4)] * 3 + [(5, 4)],
}


class Batch:
    """A batch with a cache of random values and scales, its pages in random order; the pages of a sequence's new tokens hold numbers too."""

    def __init__(self, pairs, Hq, Hkv, D, page, dtype, seed=0, spare=3, cols_more=0, behind=0, room=False):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens = [L for L, _ in pairs]
        self.cu = [sum(n for _, n in pairs[:i]) for i in range(len(pairs) + 1)]
        T = self.cu[-1] + behind
        cols = [-(-L // page) for L in self.lens]
        pages, S = sum(cols) + spare, len(pairs)
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        self.table = torch.full((S, max(1, max(cols)) + cols_more), -1, dtype=torch.int32, device="cuda")
        at = 0
        for i, n in enumerate(cols):
            self.table[i, :n] = order[at:at + n]
            at += n
        if room:   # a page more for every sequence
            self.table[range(S), cols] = order[at:at + S]
        self.p = mb.CacheParams(S=S, Hq=Hq, Hkv=Hkv, T=max(T, 1), D=D, pages=pages, page=page, table_cols=self.table.shape[1],
                                max_new=max(1, max(n for _, n in pairs)), dtype=mb.BF16 if dtype == torch.bfloat16 else mb.FP32)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        scales = lambda: torch.exp2(torch.randint(-9, -6, (pages, Hkv), generator=g, device="cuda").float())  # noqa: E731
        byte = lambda x: (100 * x).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)  # noqa: E731
        self.cache = mb.KVCache(byte(rnd(pages, Hkv, page, D)), byte(rnd(pages, Hkv, D, page)), scales(), scales())
        T = max(T, 1)
        self.Q, self.K, self.V = rnd(T, Hq, D).to(dtype), rnd(T, Hkv, D).to(dtype), rnd(T, Hkv, D).to(dtype)
        self.cud = torch.tensor(self.cu, dtype=torch.int32, device="cuda")
        self.lend = torch.tensor(self.lens, dtype=torch.int32, device="cuda")

    def values(self):
        return [x.view(torch.float8_e4m3fn).double() for x in (self.cache.k, self.cache.v)] + [x.double() for x in (self.cache.k_scale, self.cache.v_scale)]

    def append(self, cu="own"):
        mb.exact_attn_cache_append(self.p, self.K, self.V, self.cud if cu == "own" else cu, self.lend, self.table, self.cache)

    def attend(self, cu="own", **kw):
        return mb.exact_attn_cache_fwd(self.p, self.Q, self.cud if cu == "own" else cu, self.lend, self.table, self.cache, **kw)

    def check_append(self):
        want = self.values()
        ref.append(*want, self.K, self.V, self.cu, self.lens, self.table.cpu(), self.p.page)
        self.append()
        for n, a, b in zip(("k", "v", "k_scale", "v_scale"), self.values(), want):
            assert torch.equal(a.nan_to_num(1e9), b.nan_to_num(1e9)), n

    def check_attend(self, out=None):
        O, LSE = out or self.attend()
        want, tol = ref.cached(self.Q, self.cu, self.lens, self.table, *self.values(), self.p.page, self.p.scale or 1 / math.sqrt(self.p.D))
        ref.check("O", O, want["O"], tol["O"])
        ref.check("LSE", LSE, want["LSE"], tol["LSE"])
        return O, LSE


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("name", list(BATCHES))
def test_append_and_attend(name, page, D, dtype):
    """As a generation step uses them: the new tokens stored, then attended with the rest."""
    b = Batch(BATCHES[name], 4, 2, D, page, dtype)
    b.check_append()
    b.check_attend()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 1), (32, 1), (24, 1), (6, 2), (3, 3), (40, 2)])
@pytest.mark.parametrize("name", ["tokens", "drafts", "pieces"])
def test_head_layouts(name, Hq, Hkv, dtype):
    b = Batch(BATCHES[name], Hq, Hkv, 64, 32, dtype)
    b.append()
    b.check_attend()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("pairs", [[(3000, 4), (40, 4), (1800, 3)], [(2900, 9), (1, 1), (1300, 8)], [(3000, 200), (5000, 90), (7, 7)],
                                   [(2000 + 10 * i, 2) for i in range(70)]])
def test_divided_contexts(pairs, D, dtype):
    """Contexts of several workgroups, in every tile of rows; more sequences than lanes."""
    b = Batch(pairs, 8, 2, D, 64, dtype)
    b.check_append()
    b.check_attend()


@pytest.mark.parametrize("page", [16, 128])
def test_prompt_in_one_piece_is_packed_attention_of_what_is_stored(page):
    """A prompt whose keys and values are e4m3 values: stored and attended it gives what exact_attn_packed_fwd gives, within both bounds."""
    lens, D = [200, 1, 64], 64
    b = Batch([(n, n) for n in lens], 4, 2, D, page, torch.bfloat16)
    for x in (b.K, b.V):
        x.copy_(ref.e4m3(x.double()).to(x.dtype))
    b.append()
    O, LSE = b.attend()
    p = mb.PackedParams(S=3, Hq=4, Hkv=2, T=b.p.T, D=D, max_len=200)
    Op, Lp = mb.exact_attn_packed_fwd(p, b.Q, b.K, b.V, b.cud)
    _, tol = ref.packed(b.Q, b.K, b.V, b.cu, 1 / math.sqrt(D))
    ref.check("O", O, Op.double(), 2 * tol["O"])
    ref.check("LSE", LSE, Lp.double(), 2 * tol["LSE"])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
def test_token_by_token(page, D):
    """Scales that grow while a page fills: every step against the statement."""
    b = Batch([(1, 1), (page - 1, 1), (page, 1), (2 * page - 3, 1)], 2, 2, D, page, torch.bfloat16, cols_more=3)
    b.table = torch.arange(b.table.numel(), dtype=torch.int32, device="cuda").view_as(b.table)
    pages = b.table.numel()
    b.p = mb.CacheParams(**{**{f: getattr(b.p, f) for f in b.p.__dataclass_fields__}, "pages": pages})
    b.cache = mb.kv_cache(b.p)
    b.cu = list(range(5))
    for step in range(page + 3):
        b.lens = [x + (step > 0) for x in b.lens]
        b.lend = torch.tensor(b.lens, dtype=torch.int32, device="cuda")
        g = torch.Generator(device="cuda").manual_seed(step)
        for x in (b.K, b.V):
            x.copy_(torch.randn(x.shape, generator=g, device="cuda") * 1.3 ** step)
        want = b.values()
        ref.append(*want, b.K, b.V, b.cu, b.lens, b.table.cpu(), page)
        b.append(cu=None)                     # one token each
        assert all(torch.equal(x, y) for x, y in zip(b.values(), want)), step
    b.check_attend(b.attend(cu=None))


def test_magnitudes():
    """Zeros, the largest and smallest numbers, ties, and numbers that are not finite."""
    b = Batch([(16, 16)] * 6, 2, 1, 64, 16, torch.float32)
    rows = lambda i: slice(16 * i, 16 * i + 16)  # noqa: E731
    b.K[rows(0)] = 0.0
    b.K[rows(1)] *= 3.0e38 / float(b.K[rows(1)].abs().max())
    b.K[rows(2)] *= 1e-36
    b.K[rows(3)] = torch.arange(16 * 64, device="cuda").view(16, 1, 64) * 2.0 ** -9 * 448 / 1.998046875   # halves of steps
    b.K[rows(4), :, 5], b.K[rows(4), :, 6], b.K[16 * 4 + 3, :, 7] = math.inf, -math.inf, math.nan
    b.K[rows(5)] = math.nan
    b.V.copy_(b.K.roll(1, 0))
    b.check_append()


def test_nothing_else_is_touched():
    """Bytes behind the last token, pages of others, and rows behind the last sequence."""
    b = Batch([(20, 3), (40, 40), (0, 0)], 4, 2, 64, 16, torch.bfloat16, cols_more=2, behind=9)
    before = [x.clone() for x in (b.cache.k, b.cache.v, b.cache.k_scale, b.cache.v_scale)]
    b.K[b.cu[-1]:], b.V[b.cu[-1]:], b.Q[b.cu[-1]:] = math.nan, math.nan, math.nan
    b.check_append()
    used = torch.zeros(b.p.pages, dtype=torch.bool, device="cuda")
    used[b.table[0, 1].long()] = True
    used[b.table[1, :3].long()] = True
    for x, y in zip((b.cache.k, b.cache.v, b.cache.k_scale, b.cache.v_scale), before):
        assert torch.equal(x[~used], y[~used])
    pid = int(b.table[0, 1])
    assert torch.equal(b.cache.k[pid, :, 4:], before[0][pid, :, 4:]) and torch.equal(b.cache.v[pid, :, :, 4:], before[1][pid, :, :, 4:])
    O, LSE = torch.full_like(b.Q, 7.0), torch.full((4, b.p.T), 7.0, device="cuda")
    b.check_attend(b.attend(out=(O, LSE)))
    assert (O[b.cu[-1]:] == 7.0).all() and (LSE[:, b.cu[-1]:] == 7.0).all()


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_places_without_tokens_hold_anything(page, dtype):
    """NaN bytes behind the last token and NaN scales of pages that no length reaches do not count."""
    b = Batch([(page + 3, 1), (5, 2), (3 * page, 3), (2 * page + page // 2, 1)], 4, 2, 64, page, dtype, cols_more=1)
    want = b.check_attend()
    for i, L in enumerate(b.lens):
        for col in range(b.table.shape[1]):
            pid = int(b.table[i, col])
            lo = max(0, min(page, L - col * page))
            if pid >= 0:
                b.cache.k[pid, :, lo:] = 127
                b.cache.v[pid, :, :, lo:] = 255
    free = [x for x in range(b.p.pages) if x not in set(b.table.flatten().tolist())]
    b.cache.k[free], b.cache.v[free], b.cache.k_scale[free], b.cache.v_scale[free] = 127, 127, math.nan, math.nan
    b.table[:, -1] = free[0]   # past every length
    assert all(torch.equal(x, y) for x, y in zip(b.attend(), want))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_missing_pages_and_rows_without_keys(dtype):
    """Entries outside the cache are pages without tokens; more new tokens than the length has rows at positions below 0; a sequence longer
    than its table."""
    b = Batch([(100, 2), (50, 3), (2, 5), (0, 3), (70, 70), (400, 4)], 4, 2, 64, 16, dtype)
    b.table[0, 1], b.table[0, 4], b.table[1, :] = -1, b.p.pages, -7
    b.table[4, 2] = 1 << 30
    b.table = b.table[:, :20].contiguous()
    b.p = mb.CacheParams(**{**{f: getattr(b.p, f) for f in b.p.__dataclass_fields__}, "table_cols": 20})
    b.check_append()
    O, LSE = b.check_attend()
    for rows in (slice(b.cu[1], b.cu[2]), slice(b.cu[2], b.cu[2] + 3), slice(b.cu[3], b.cu[4])):
        assert (O[rows] == 0).all() and (LSE[:, rows] == -math.inf).all()


def test_shared_pages():
    """Two sequences that read the same first pages."""
    b = Batch([(100, 1), (90, 1), (100, 1)], 4, 2, 64, 32, torch.bfloat16)
    b.table[1, :2] = b.table[0, :2]
    b.check_attend()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("max_new", [0, 1, 7, 5000])
@pytest.mark.parametrize("pairs", [[(300, 70), (90, 1), (33, 33)], [(3000, 70), (90, 1), (1500, 150)], [(20 + i, 1 + i % 40) for i in range(40, 110)]])
def test_the_bound_on_new_tokens_is_a_hint(pairs, max_new, dtype):
    b = Batch(pairs, 8, 2, 64, 32, dtype)
    b.p = mb.CacheParams(**{**{f: getattr(b.p, f) for f in b.p.__dataclass_fields__}, "max_new": max_new})
    b.check_append()
    b.check_attend()


def test_strides_and_no_lse():
    b = Batch([(300, 20), (90, 1)], 4, 2, 64, 32, torch.bfloat16)
    fused = torch.cat([b.Q, b.K, b.V], 1)
    other = Batch([(300, 20), (90, 1)], 4, 2, 64, 32, torch.bfloat16)
    b.append()
    want = b.attend()
    other.Q, other.K, other.V = fused[:, :4], fused[:, 4:6], fused[:, 6:].transpose(0, 1).contiguous().transpose(0, 1)
    other.append()
    assert torch.equal(b.cache.k, other.cache.k) and torch.equal(b.cache.v, other.cache.v)
    O = torch.zeros(4, b.p.T, 64, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    got = other.attend(out=(O, torch.zeros_like(want[1])))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_many_sequences_and_long_ones():
    """More sequences than a wave has lanes, ragged; and contexts that are divided among workgroups."""
    b = Batch([((37 * i) % 211, min((37 * i) % 211, 1 + i % 2)) for i in range(300)], 2, 1, 64, 16, torch.bfloat16)
    b.check_append()
    b.check_attend()
    b = Batch([(20000, 1), (7, 1), (9000, 2)], 4, 1, 64, 64, torch.bfloat16)
    b.check_append()
    b.check_attend()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_captured_into_graphs(dtype):
    """Two graphs of a step of generation, replayed in turn; lengths, tokens and tables are read at replay."""
    cases = []
    for seed, pairs in ((1, [(700, 1), (30, 1), (65, 1)]), (2, [(64, 1), (1200, 1)])):
        a, e = (Batch(pairs, 4, 2, 64, 64, dtype, seed=seed, cols_more=1, room=True) for _ in range(2))
        a.append()
        a.attend()
        e.append()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            a.append()
            out = a.attend()
        cases.append((graph, a, e, out))
    for _ in range(4):
        for graph, a, e, out in cases:
            for b in (a, e):
                b.lend.add_(1)
                for x in (b.Q, b.K, b.V):
                    x.mul_(1.5)
            graph.replay()
            e.append()
            want = e.attend()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(out, want))
            assert torch.equal(a.cache.k, e.cache.k) and torch.equal(a.cache.v, e.cache.v)


def test_on_other_streams_and_the_same_bits():
    b = Batch([(3000, 2), (500, 1)], 8, 2, 128, 64, torch.bfloat16)
    b.append()
    want = b.attend()
    torch.cuda.synchronize()
    got = []
    for st in [torch.cuda.Stream() for _ in range(2)]:
        with torch.cuda.stream(st):
            got.append(b.attend())
    torch.cuda.synchronize()
    for g in got:
        assert torch.equal(g[0], want[0]) and torch.equal(g[1], want[1])


def test_offsets_past_32_bits():
    """A cache of more than 4 GB, with tokens in its last pages."""
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 30 GB of device memory")
    p = mb.CacheParams(S=1, Hq=2, Hkv=2, T=1, D=128, pages=150_000, page=128, table_cols=3, max_new=1)
    cache = mb.kv_cache(p)
    assert cache.k.numel() > 1 << 32
    small = Batch([(300, 1)], 2, 2, 128, 128, torch.bfloat16, spare=0)
    at = torch.tensor([149_999, 0, 140_001], device="cuda")
    src = small.table[0].long()
    for n in ("k", "v", "k_scale", "v_scale"):
        getattr(cache, n)[at] = getattr(small.cache, n)[src]
    table = at.to(torch.int32)[None].contiguous()
    mb.exact_attn_cache_append(p, small.K, small.V, None, small.lend, table, cache)
    got = mb.exact_attn_cache_fwd(p, small.Q, None, small.lend, table, cache)
    small.append()
    want = small.attend()
    for n in ("k", "v", "k_scale", "v_scale"):
        assert torch.equal(getattr(cache, n)[at], getattr(small.cache, n)[src])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
