"""What the operators of exact attention over packed sequences and over an 8-bit cache are measured on: calls that a user's
program makes through `paper_2509_10406_amd.binding`, and the same operators in plain torch operations.

A case is a dict of plain values.  Its `path` says which calls one pass makes:
  "prompt"  exact_attn_packed_fwd: causal attention over whole prompts of different lengths, packed one after the other
  "train"   exact_attn_packed_fwd + exact_attn_packed_bwd: the same in a training step, with its gradients
  "store"   exact_attn_cache_append: new tokens' keys and values into a paged cache of 8-bit values
  "decode"  exact_attn_cache_fwd: the new tokens' queries against the cache
  "step"    exact_attn_cache_append + exact_attn_cache_fwd: a layer's attention in one step of generation
The other values: S sequences, heads Hq and Hkv, head dimension D, dtype, and
  prompt, train: `lens`, the spread of the lengths ("even": around T / S, "mixed": over their logarithm, with one-token and
      empty sequences among them, "one_long": the first has about half of the tokens), T tokens in all
  store, decode, step: pages of `page` tokens; contexts of `ctx` tokens at the most (the shortest a thirtieth of that, or all
      alike where `lens` is "even"), of which each sequence's last 1 .. `new` are the new ones

The cache of a sequence is the pages that its row of the table names, in order.  A page holds, per key/value head, `page` keys
as [page, D] and values as [D, page] of e4m3, and a scale for each of the two: the stored value stands for itself times the
scale.  The scale is the least power of two, 2^-100 at the least, by which the largest finite magnitude put into the page so
far stays within 448; when a new token raises it, what the page holds is rounded again.  Query i of a sequence with n new
tokens and a length of L (the new ones included) attends to the keys at positions 0 .. L - n + i.
"""
import math

import torch

own = False

MOST = 448.0          # the largest e4m3 value
LEAST_EXPONENT = -100


def _case(name, path, **kw):
    c = dict(name=name, path=path, S=1, Hq=8, Hkv=8, D=64, dtype="bf16", lens="mixed")
    c.update(dict(T=64) if path in ("prompt", "train") else dict(page=64, ctx=1024, new=1))
    c.update(kw)
    return c


def listed():
    return [
        # three short questions to a small model at once: latency counts
        _case("prompt_few", "prompt", S=3, T=70, Hq=4, Hkv=2, D=64),
        # a serving engine's prefill batch, from one token to some three thousand, grouped heads
        _case("prompt_batch", "prompt", S=16, T=12289, Hq=32, Hkv=8, D=128),
        # long documents beside short ones
        _case("prompt_long", "prompt", S=4, T=16384, Hq=32, Hkv=8, D=128, lens="one_long"),
        # gradients checked or a method debugged in fp32
        _case("train_few_fp32", "train", S=5, T=1501, Hq=4, Hkv=2, D=64, dtype="fp32"),
        # instruction tuning of a small model: many short conversations, packed
        _case("train_batch", "train", S=40, T=16000, Hq=16, Hkv=16, D=64, lens="even"),
        # long-context training with grouped heads: the largest call
        _case("train_long", "train", S=3, T=16384, Hq=32, Hkv=8, D=128, lens="one_long"),
        # one step of generation for many requests: a token each into the cache
        _case("store_tokens", "store", S=128, ctx=4000, Hkv=8, Hq=32, D=128, page=64),
        # whole prompts into the cache
        _case("store_prompts", "store", S=8, ctx=4096, new=4096, Hkv=8, Hq=32, D=128, page=64),
        # one request of a small model
        _case("decode_one", "decode", S=1, ctx=1000, Hq=8, Hkv=8, D=64, page=16, lens="even"),
        # a serving batch of ragged contexts, its new tokens stored and attended
        _case("step_batch", "step", S=64, ctx=8192, Hq=32, Hkv=8, D=128, page=64),
        # few requests over very long contexts
        _case("decode_long", "decode", S=2, ctx=131072, Hq=32, Hkv=8, D=128, page=128, lens="even"),
        # prompts that are taken in pieces, and drafts that are checked: several new tokens on a context
        _case("decode_pieces", "decode", S=8, ctx=4096, new=300, Hq=16, Hkv=4, D=128, page=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the ranges above: 1 to 64 sequences (128 where single tokens are stored), up to 16k new tokens, contexts to 128k,
    1 to 32 heads, both head dimensions and types, pages of 16 to 128."""
    while True:
        path = rng.choice(["prompt", "train", "store", "decode", "step"])
        group = rng.choice([1, 2, 4, 4, 8])
        Hkv = _log_int(rng, 1, 16)
        kw = dict(Hkv=Hkv, Hq=Hkv * group, D=rng.choice([64, 128]), dtype=rng.choice(["bf16", "bf16", "bf16", "fp32"]))
        if kw["Hq"] > 32:
            continue
        if path in ("prompt", "train"):
            kw["T"] = _log_int(rng, 24, 16384 if kw["dtype"] == "bf16" else 4096)
            kw["S"] = min(_log_int(rng, 1, 64), kw["T"])
            kw["lens"] = rng.choice(["even", "mixed", "one_long"])
            if kw["lens"] == "one_long" and kw["S"] == 1:
                continue
        else:
            kw["page"] = rng.choice([16, 32, 64, 128])
            kw["ctx"] = _log_int(rng, 20, 131072)
            kw["S"] = _log_int(rng, 1, 128 if path == "store" else 64)
            kw["lens"] = rng.choice(["even", "mixed"])
            kw["new"] = rng.choice([1, 1, 1, _log_int(rng, 2, 512)]) if path != "store" else rng.choice([1, _log_int(rng, 2, 4096)])
            kw["new"] = min(kw["new"], kw["ctx"])
        c = _case("", path, **kw)
        del c["name"]
        if path in ("prompt", "train"):
            # the plain form's scores of all pairs: 4 x 32 x 8192^2 at the most (fp32 products take a multiple of the time)
            longest = max(_lengths(c))
            if c["S"] * c["Hq"] * longest * longest * (4 if c["dtype"] == "fp32" else 1) > 4 * 32 * 8192 * 8192:
                continue
            if path == "train" and work(c)["flops"] > work(listed()[5])["flops"]:
                continue
            if path == "prompt" and work(c)["flops"] > work(listed()[2])["flops"]:
                continue
        else:
            tokens = c["S"] * c["ctx"]
            if tokens * c["Hkv"] * c["D"] > 2 * 131072 * 8 * 128 or c["S"] * c["new"] * c["Hkv"] * c["D"] > 32768 * 8 * 128:
                continue
            if path != "store" and c["S"] * c["new"] * c["Hq"] * c["ctx"] > 8 * 300 * 16 * 4096 * (1 if c["dtype"] == "bf16" else 0.25):
                continue
        return c


def _spread(c, i, S):
    """A fixed pseudo-random number of [0, 1) for the i-th sequence of a case."""
    return (0.6180339887498949 * (i + 1) + 0.37 * S) % 1.0


def _lengths(c):
    """Lengths of the packed sequences, T tokens in all."""
    S, T = c["S"], c["T"]
    if c["lens"] == "even":
        w = [0.7 + 0.6 * _spread(c, i, S) for i in range(S)]
    elif c["lens"] == "one_long":
        w = [1.0] + [2.0 * _spread(c, i, S) / S for i in range(S - 1)]
    else:
        w = [math.exp(3.0 * _spread(c, i, S)) for i in range(S)]
    lens = [int(T * x / sum(w)) for x in w]
    if c["lens"] == "mixed" and S >= 5:
        lens[1], lens[2] = 0, 1
    at = max(range(S), key=lambda i: lens[i])
    lens[at] += T - sum(lens)
    return lens


def _contexts(c):
    """(length with the new tokens, new tokens) of every sequence of a cache case."""
    S, got = c["S"], []
    for i in range(S):
        u = _spread(c, i, S)
        L = c["ctx"] if c["lens"] == "even" else max(1, int(c["ctx"] * math.exp(-math.log(30.0) * u)))
        n = 1 if c["new"] == 1 else max(1, int(c["new"] * (1.0 - 0.7 * u)))
        if c["path"] == "store" and c["new"] > 1 and i % 4 != 3:
            L = n                      # a prompt from its first token on; every fourth one follows an earlier piece
        got.append((max(L, n), n))
    return got


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _activations(g, n, heads, D):
    """Projections of token embeddings that are drawn from a mixture: as in a layer, the heads, and Q, K and V, of a token share it.
    Returns [n, H, D] for every count of heads."""
    E = 256
    centres = torch.randn(max(16, min(512, n // 64)), E, generator=g, device="cuda")
    emb = centres[torch.randint(0, centres.shape[0], (n,), generator=g, device="cuda")]
    emb = emb + 0.5 * torch.randn(n, E, generator=g, device="cuda")
    return [(emb @ (torch.randn(E, H * D, generator=g, device="cuda") / math.sqrt(1.25 * E))).view(n, H, D) for H in heads]


def _quantise(x, scale):
    """fp32 values -> e4m3 bytes for a power of two that keeps them within 448."""
    return (x / scale).to(torch.float8_e4m3fn)


def _power_of_two(amax):
    """The least power of two by which values up to amax stay within 448 = 0.875 * 2^9."""
    m, e = torch.frexp(amax)
    e = torch.where(m > 0.875, e - 8, e - 9)
    return torch.ldexp(torch.ones_like(amax), e.clamp(min=LEAST_EXPONENT))


def prepare(case, seed):
    """The activations of a batch and what the program has in hand with them: offsets of the sequences, or the cache with
    its table and lengths, as earlier calls have left it."""
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    t, s = _dtype(c), {"case": c}
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    if c["path"] in ("prompt", "train"):
        lens = _lengths(c)
        s["Q"], s["K"], s["V"] = (x.to(t).contiguous() for x in _activations(g, c["T"], (c["Hq"], c["Hkv"], c["Hkv"]), c["D"]))
        s["cu"], s["max_len"] = ints([0] + [sum(lens[: i + 1]) for i in range(c["S"])]), max(lens)
        if c["path"] == "train":
            s["dO"] = torch.randn(c["T"], c["Hq"], c["D"], generator=g, device="cuda").to(t)
        return s
    ctx, page, Hkv, D = _contexts(c), c["page"], c["Hkv"], c["D"]
    cols = [-(-L // page) for L, _ in ctx]
    need = sum(cols)
    pages = need + max(1, need // 16)  # some are free
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((c["S"], max(cols)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(cols):
        table[i, :n] = order[at:at + n]
        at += n
    s["table"], s["lens"], s["max_new"] = table, ints([L for L, _ in ctx]), max(n for _, n in ctx)
    s["cu"] = ints([0] + [sum(n for _, n in ctx[: i + 1]) for i in range(c["S"])])
    T = sum(n for _, n in ctx)
    s["Q"], s["newK"], s["newV"] = (x.to(t).contiguous() for x in _activations(g, T, (c["Hq"], Hkv, Hkv), D))
    # what earlier calls have stored: every page full of values of its own scale (pages that are to be begun, too: recycled ones)
    for name in "KV":
        x = torch.empty(pages, Hkv, page, D, device="cuda")
        step = max(1, (1 << 26) // (Hkv * page * D))
        for p0 in range(0, pages, step):
            n = min(step, pages - p0)
            x[p0:p0 + n] = _activations(g, n * page, (Hkv,), D)[0].view(n, page, Hkv, D).transpose(1, 2)
        scale = _power_of_two(x.abs().amax((2, 3)))
        q = _quantise(x, scale[:, :, None, None])
        s[name.lower()] = (q if name == "K" else q.view(torch.uint8).transpose(2, 3)).contiguous().view(torch.uint8)
        s[name.lower() + "_scale"] = scale
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------------
def _rows(cu, T):
    """(sequence, place in it) of every packed row."""
    at = torch.arange(T, device=cu.device)
    seq = torch.searchsorted(cu[1:].long(), at, right=True)
    return seq, at - cu[seq].long()


def _padded(x, cu, longest):
    """[T, H, D] -> fp32 [S, H, longest, D], zeros behind a sequence's end."""
    at = torch.arange(longest, device=cu.device)
    lens = (cu[1:] - cu[:-1]).long()
    i = (cu[:-1, None].long() + at).clamp(max=x.shape[0] - 1)
    return (x[i].float() * (at < lens[:, None])[:, :, None, None]).transpose(1, 2).contiguous()


def _softmax_(s, hidden):
    """(weights before the division, their sum, the logarithm of the softmax's normaliser) of scores, in place."""
    s.masked_fill_(hidden, -math.inf)
    m = s.amax(-1, keepdim=True).clamp(min=-3.0e38)
    s.sub_(m).exp_()
    l = s.sum(-1, keepdim=True)
    return s, l, (m + l.log()).squeeze(-1)


def _plain_packed(s):
    c, cu, L = s["case"], s["cu"], s["max_len"]
    t, G, scale = _dtype(c), c["Hq"] // c["Hkv"], 1.0 / math.sqrt(c["D"])
    seq, at = _rows(cu, c["T"])
    back = lambda x: x.transpose(1, 2)[seq, at].to(t)  # noqa: E731
    q = _padded(s["Q"], cu, L)
    k, v = (_padded(s[n], cu, L).repeat_interleave(G, 1) for n in "KV")
    pos = torch.arange(L, device=cu.device)
    hidden = (pos[None, :] > pos[:, None])[None, None]   # a key behind the end of a sequence is behind all its queries
    p, l, lse = _softmax_(torch.matmul(q, k.transpose(2, 3)).mul_(scale), hidden)
    o = torch.matmul(p, v) / l
    out = {"O": back(o), "LSE": lse.transpose(1, 2)[seq, at].t().contiguous()}
    if c["path"] == "prompt":
        return out
    g = _padded(s["dO"], cu, L)
    p.div_(l)
    dv = torch.matmul(p.transpose(2, 3), g)
    ds = torch.matmul(g, v.transpose(2, 3)).sub_((g * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    group = lambda x: x.unflatten(1, (c["Hkv"], G)).sum(2)  # noqa: E731
    out["dQ"] = back(torch.matmul(ds, k))
    out["dK"], out["dV"] = back(group(torch.matmul(ds.transpose(2, 3), q))), back(group(dv))
    return out


def _plain_store(s):
    c, page, table, cu = s["case"], s["case"]["page"], s["table"].long(), s["cu"].long()
    n, L = cu[1:] - cu[:-1], s["lens"].long()
    first = L - n
    C = s["max_new"] // page + 2                                         # pages that a sequence's new tokens touch, at the most
    col = first[:, None] // page + torch.arange(C, device=cu.device)
    used = (col * page < L[:, None]) & (n > 0)[:, None]
    seq = torch.arange(c["S"], device=cu.device)[:, None].expand_as(col)[used]
    pos = col[used][:, None] * page + torch.arange(page, device=cu.device)   # [touched pages, page]
    pid = table[seq, col[used]]
    new = (pos >= first[seq][:, None]) & (pos < L[seq][:, None])
    held = pos < first[seq][:, None]
    row = (cu[seq][:, None] + pos - first[seq][:, None]).clamp(0, s["newK"].shape[0] - 1)
    for name in "kv":
        cache, scales = s[name], s[name + "_scale"]
        x = s["new" + name.upper()][row].float().transpose(1, 2)        # [pages, Hkv, page, D]
        mark = new[:, None, :, None]
        amax = torch.where(mark & x.isfinite(), x.abs(), 0.0).amax((2, 3))
        old = torch.where(held.any(1)[:, None], scales[pid], 0.0)
        scale = torch.maximum(_power_of_two(amax), old)
        was = cache[pid] if name == "k" else cache[pid].transpose(2, 3)
        again = _quantise(was.contiguous().view(torch.float8_e4m3fn).float() * old[:, :, None, None], scale[:, :, None, None]).view(torch.uint8)
        fresh = _quantise(torch.where(x.isfinite(), x, math.nan), scale[:, :, None, None]).view(torch.uint8)
        now = torch.where(mark, fresh, torch.where(held[:, None, :, None], again, was))
        cache[pid] = now if name == "k" else now.transpose(2, 3).contiguous()
        scales[pid] = scale


def _plain_decode(s):
    c, page, cu = s["case"], s["case"]["page"], s["cu"]
    t, G, D, S = _dtype(c), c["Hq"] // c["Hkv"], c["D"], c["S"]
    table = s["table"].long()
    keys = table.shape[1] * page
    pid = table.clamp(min=0)
    k = s["k"][pid].view(torch.float8_e4m3fn).float() * s["k_scale"][pid][..., None, None]     # [S, pages, Hkv, page, D]
    v = s["v"][pid].view(torch.float8_e4m3fn).float() * s["v_scale"][pid][..., None, None]     # [S, pages, Hkv, D, page]
    k = k.permute(0, 2, 4, 1, 3).reshape(S, c["Hkv"], D, keys)
    v = v.permute(0, 2, 1, 4, 3).reshape(S, c["Hkv"], keys, D)
    q = _padded(s["Q"], cu, s["max_new"])                                                       # [S, Hq, new, D]
    n, L = (cu[1:] - cu[:-1]).long(), s["lens"].long()
    at, pos = torch.arange(s["max_new"], device=cu.device), torch.arange(keys, device=cu.device)
    last = (L - n)[:, None] + torch.minimum(at, n[:, None] - 1)                                 # of every query
    hidden = (pos > last[:, :, None])[:, None, None]
    v = torch.where((pos < L[:, None])[:, None, :, None], v, 0.0)                               # nothing of pages that end later
    q = q.unflatten(1, (c["Hkv"], G))
    sc = torch.matmul(q.flatten(2, 3), k).mul_(1.0 / math.sqrt(D)).unflatten(2, (G, -1))
    p, l, lse = _softmax_(sc, hidden)
    o = (torch.matmul(p.flatten(2, 3), v).unflatten(2, (G, -1)) / l).flatten(1, 2)
    seq, row = _rows(cu, s["Q"].shape[0])
    return {"O": o.transpose(1, 2)[seq, row].to(t), "LSE": lse.flatten(1, 2).transpose(1, 2)[seq, row].t().contiguous()}


def _stored(s):
    return {n: s[n].view(torch.float8_e4m3fn) for n in "kv"} | {n: s[n] for n in ("k_scale", "v_scale")}


def run(state):
    s, c = state, state["case"]
    path = c["path"]
    if not own:
        out = {}
        if path in ("prompt", "train"):
            return _plain_packed(s)
        if path in ("store", "step"):
            _plain_store(s)
            out = _stored(s)
        return out if path == "store" else out | _plain_decode(s)
    from paper_2509_10406_amd import binding as mb

    dtype = mb.BF16 if c["dtype"] == "bf16" else mb.FP32
    if path in ("prompt", "train"):
        if "p" not in s:
            s["p"] = mb.PackedParams(S=c["S"], Hq=c["Hq"], Hkv=c["Hkv"], T=c["T"], D=c["D"], max_len=s["max_len"], dtype=dtype, grad_dtype=dtype)
        p = s["p"]
        O, LSE = mb.exact_attn_packed_fwd(p, s["Q"], s["K"], s["V"], s["cu"])
        if path == "prompt":
            return {"O": O, "LSE": LSE}
        dQ, dK, dV = mb.exact_attn_packed_bwd(p, s["Q"], s["K"], s["V"], s["cu"], O, LSE, s["dO"])
        return {"O": O, "LSE": LSE, "dQ": dQ, "dK": dK, "dV": dV}
    if "p" not in s:
        s["p"] = mb.CacheParams(S=c["S"], Hq=c["Hq"], Hkv=c["Hkv"], T=s["Q"].shape[0], D=c["D"], pages=s["k"].shape[0], page=c["page"],
                                table_cols=s["table"].shape[1], max_new=s["max_new"], dtype=dtype)
        s["cache"] = mb.KVCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
    p, out = s["p"], {}
    if path in ("store", "step"):
        mb.exact_attn_cache_append(p, s["newK"], s["newV"], s["cu"], s["lens"], s["table"], s["cache"])
        out = _stored(s)
    if path == "store":
        return out
    O, LSE = mb.exact_attn_cache_fwd(p, s["Q"], s["cu"], s["lens"], s["table"], s["cache"])
    return out | {"O": O, "LSE": LSE}


def work(case):
    """Inputs read once and outputs written once; 2 products forward and 5 backward over the pairs that are attended.  Of a cache the
    keys and values of the sequences' own tokens, and the scales of their pages."""
    c = case
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    es = 2 if c["dtype"] == "bf16" else 4
    if c["path"] in ("prompt", "train"):
        lens = _lengths(c)
        pairs = sum(n * (n + 1) // 2 for n in lens) * Hq
        rows = 2 * c["T"] * (Hq + Hkv) * D * es + c["T"] * Hq * 4       # Q, O and K, V; the logarithms
        if c["path"] == "prompt":
            return {"bytes": rows, "flops": 4 * pairs * D}
        return {"bytes": rows + c["T"] * Hq * D * es + c["T"] * (Hq + 2 * Hkv) * D * es, "flops": 14 * pairs * D}
    ctx = _contexts(c)
    T, pages = sum(n for _, n in ctx), sum(-(-L // c["page"]) for L, _ in ctx)
    got = {"bytes": 0, "flops": 0}
    if c["path"] != "decode":
        touched = sum((L - 1) // c["page"] - (L - n) // c["page"] + 1 for L, n in ctx)
        got["bytes"] += 2 * T * Hkv * D * (es + 1) + touched * (4 + 8 * Hkv)
    if c["path"] != "store":
        tokens = sum(L for L, _ in ctx)
        pairs = sum(n * (L - n) + n * (n + 1) // 2 for L, n in ctx) * Hq
        got["bytes"] += 2 * tokens * Hkv * D + pages * (4 + 8 * Hkv) + 2 * T * Hq * D * es + T * Hq * 4
        got["flops"] += 4 * pairs * D
    return got


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------------
def _attend64(q, k, v, first, g=None):
    """One head of one sequence: queries at positions first .. of keys 0 ..; with g, its gradients too."""
    scale = 1.0 / math.sqrt(q.shape[1])
    z = q @ k.T * scale
    z = torch.where(torch.arange(k.shape[0], device=q.device) <= first + torch.arange(q.shape[0], device=q.device)[:, None], z, -math.inf)
    lse = torch.logsumexp(z, 1)
    w = torch.exp(z - lse[:, None])
    o = w @ v
    if g is None:
        return o, lse
    dz = w * (g @ v.T - (w * (g @ v.T)).sum(1, keepdim=True))
    return o, lse, dz @ k * scale, dz.T @ q * scale, w.T @ g


def _exact_packed(s):
    c = s["case"]
    G, cu = c["Hq"] // c["Hkv"], s["cu"].tolist()
    Q, K, V = (s[n].double() for n in "QKV")
    out = {"O": torch.zeros_like(Q), "LSE": torch.zeros(c["Hq"], c["T"], dtype=torch.float64, device=Q.device)}
    if c["path"] == "train":
        out.update(dQ=torch.zeros_like(Q), dK=torch.zeros_like(K), dV=torch.zeros_like(V))
    for a, b in zip(cu[:-1], cu[1:]):
        if a == b:
            continue
        for h in range(c["Hq"]):
            hk = h // G
            if c["path"] == "prompt":
                out["O"][a:b, h], out["LSE"][h, a:b] = _attend64(Q[a:b, h], K[a:b, hk], V[a:b, hk], 0)
                continue
            o, lse, dq, dk, dv = _attend64(Q[a:b, h], K[a:b, hk], V[a:b, hk], 0, s["dO"][a:b, h].double())
            out["O"][a:b, h], out["LSE"][h, a:b], out["dQ"][a:b, h] = o, lse, dq
            out["dK"][a:b, hk] += dk
            out["dV"][a:b, hk] += dv
    return out


def _e4m3_of(x):
    """The nearest e4m3 value, ties to even, for |x| <= 448: steps of 2^-3 of the binade, 2^-9 below 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_store(s):
    """The caches as (value, scale) per page, in 64 bits: page after page."""
    c, page = s["case"], s["case"]["page"]
    cu, lens, table = s["cu"].tolist(), s["lens"].tolist(), s["table"].tolist()
    out = {n: s[n].view(torch.float8_e4m3fn).double() for n in "kv"}
    out.update({n: s[n].double() for n in ("k_scale", "v_scale")})
    for i in range(c["S"]):
        n, L = cu[i + 1] - cu[i], lens[i]
        for col in range((L - n) // page, -(-L // page)) if n else ():
            a, b = max(L - n, col * page), min(L, (col + 1) * page)
            lo, hi, pid, row = a - col * page, b - col * page, table[i][col], cu[i] + a - (L - n)
            for name in "kv":
                x = s["new" + name.upper()][row:row + b - a].double().transpose(0, 1)          # [Hkv, tokens, D]
                val = out[name][pid] if name == "k" else out[name][pid].transpose(1, 2)        # [Hkv, page, D]
                old = out[name + "_scale"][pid].clone() if lo else torch.zeros(c["Hkv"], dtype=torch.float64, device=x.device)
                top = x.abs().amax((1, 2))
                least = torch.exp2(torch.ceil(torch.log2(top / MOST)).clamp(min=LEAST_EXPONENT))
                scale = torch.maximum(least, old)
                val[:, :lo] = _e4m3_of(val[:, :lo] * (old / scale)[:, None, None])
                val[:, lo:hi] = _e4m3_of(x / scale[:, None, None])
                out[name + "_scale"][pid] = scale
    return out


def _exact_decode(s, st):
    c, page = s["case"], s["case"]["page"]
    G, cu, lens, table = c["Hq"] // c["Hkv"], s["cu"].tolist(), s["lens"].tolist(), s["table"]
    T = s["Q"].shape[0]
    out = {"O": torch.zeros(T, c["Hq"], c["D"], dtype=torch.float64, device=table.device),
           "LSE": torch.zeros(c["Hq"], T, dtype=torch.float64, device=table.device)}
    for i in range(c["S"]):
        a, b, L = cu[i], cu[i + 1], lens[i]
        pid = table[i, : -(-L // page)].long()
        for hk in range(c["Hkv"]):
            k = (st["k"][pid, hk].double() * st["k_scale"][pid, hk].double()[:, None, None]).flatten(0, 1)[:L]
            v = (st["v"][pid, hk].double() * st["v_scale"][pid, hk].double()[:, None, None]).transpose(1, 2).flatten(0, 1)[:L]
            for h in range(hk * G, hk * G + G):
                out["O"][a:b, h], out["LSE"][h, a:b] = _attend64(s["Q"][a:b, h].double(), k, v, L - (b - a))
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["path"] in ("prompt", "train"):
        return _exact_packed(s)
    st = _stored(s) if case["path"] == "decode" else _exact_store(s)
    out = {} if case["path"] == "decode" else st
    return out if case["path"] == "store" else out | _exact_decode(s, st)
