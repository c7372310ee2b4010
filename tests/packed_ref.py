"""64-bit statements of attention over packed sequences and over the paged cache, for the tests, with bounds on the rounding of the
library's results: sums of the magnitudes that each rounding applies to.  Half a step of a type is finfo(t).eps / 2 of the value."""
import math

import torch

STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24, torch.float64: 0.0}


def head(q, k, v, first, scale, g=None, o_used=None):
    """One head of one sequence, 64 bits: queries at positions first .. of keys 0 ...  Returns dicts of results and of what their
    rounding is relative to.  o_used: the rounded O that the backward is given."""
    n, m = q.shape[0], k.shape[0]
    at = first + torch.arange(n, device=q.device)
    seen = torch.arange(m, device=q.device)[None, :] <= at[:, None]
    z = torch.where(seen, q @ k.T * scale, -math.inf)
    lse = torch.logsumexp(z, 1) if m else torch.full((n,), -math.inf, dtype=q.dtype, device=q.device)
    w = torch.where(seen & (lse > -math.inf)[:, None], torch.exp(z - torch.where(lse > -math.inf, lse, 0.0)[:, None]), 0.0)
    mag = torch.where(seen, q.abs() @ k.abs().T * scale, 0.0)
    size = mag.amax(1) if m else torch.zeros_like(lse)  # the largest score's terms, for what 32-bit sums of D products lose
    got = {"O": w @ v, "LSE": lse}
    err = {"size": size, "P|v|": w @ v.abs()}
    if g is None:
        return got, err
    dp = g @ v.T
    delta = (w * dp).sum(1, keepdim=True)
    ds = w * (dp - delta)
    got.update(dQ=ds @ k * scale, dK=ds.T @ q * scale, dV=w.T @ g)
    wide = w * (g.abs() @ v.abs().T + (g * got["O"]).abs().sum(1, keepdim=True))  # what 32-bit roundings in dS are relative to
    doff = (g * o_used).abs().sum(1, keepdim=True) if o_used is not None else torch.zeros_like(delta)
    err.update({"dS|k|": ds.abs() @ k.abs() * scale, "dS|q|": ds.abs().T @ q.abs() * scale, "P|g|": w.T @ g.abs(),
                "wide|k|": wide @ k.abs() * scale, "wide|q|": wide.T @ q.abs() * scale, "wide_P|g|": (w * size[:, None]).T @ g.abs(),
                "Poff|k|": (w * doff) @ k.abs() * scale, "Poff|q|": (w * doff).T @ q.abs() * scale})
    return got, err


def bounds(got, err, D, n, dtype, grad_dtype=None):
    """Bounds on |result - got|.  32-bit parts: a score of D products is off by at most (D + 2) 2^-24 of its terms' size, its exponential
    by that and 4 steps (exp2, the product with log2 e, the maximum, the normaliser), sums of n terms by n 2^-24 (taken as 32 steps
    at least).  bf16: P and dS are rounded once, half a step each, and so are the results; the backward's sum dO.O uses the O it was
    given, off by half a step.  2 on the 32-bit parts covers the second order."""
    f = 2.0 ** -24
    eps = 2 * f * ((D + 2) * err["size"] + 8 + max(32, n))
    b = {"LSE": eps + 4 * f * got["LSE"].abs().clamp(max=1e30)}
    half = STEP[dtype] if dtype == torch.bfloat16 else 0.0
    b["O"] = (eps[:, None] + half) * err["P|v|"] + STEP[dtype] * got["O"].abs()
    if "dQ" in got:
        gh, top = STEP[grad_dtype], 2 * f * ((D + 2) * float(err["size"].max()) + D + 8 + max(32, n))
        b["dQ"] = half * err["dS|k|"] + (STEP[dtype] + f * D) * err["Poff|k|"] + top * err["wide|k|"] + gh * got["dQ"].abs()
        b["dK"] = half * err["dS|q|"] + (STEP[dtype] + f * D) * err["Poff|q|"] + top * err["wide|q|"] + gh * got["dK"].abs()
        b["dV"] = half * err["P|g|"] + top * (err["P|g|"] + err["wide_P|g|"]) + gh * got["dV"].abs()
    # a result that came through two roundings relative to one another: 1 % for their product terms; nothing below the smallest normals
    return {k: 1.01 * x + 1e-35 for k, x in b.items()}


def packed(Q, K, V, cu, scale, dO=None, O=None, grad_dtype=None):
    """Results and bounds over all sequences and heads.  Rows of no sequence are NaN in both."""
    T, Hq, D = Q.shape
    Hkv, dtype = K.shape[1], Q.dtype
    G = Hq // Hkv
    nan = lambda *s: torch.full(s, math.nan, dtype=torch.float64, device=Q.device)  # noqa: E731
    names = ("O", "LSE") + (("dQ", "dK", "dV") if dO is not None else ())
    shape = {"O": (T, Hq, D), "LSE": (Hq, T), "dQ": (T, Hq, D), "dK": (T, Hkv, D), "dV": (T, Hkv, D)}
    got, tol = ({n: nan(*shape[n]) for n in names} for _ in range(2))
    d = lambda x, a, b, h: x[a:b, h].double()  # noqa: E731
    for a, b in zip(cu[:-1], cu[1:]):
        if a >= b:
            continue
        for n in names[3:]:
            got[n][a:b], tol[n][a:b] = 0.0, 0.0
        for h in range(Hq):
            hk = h // G
            r, e = head(d(Q, a, b, h), d(K, a, b, hk), d(V, a, b, hk), 0, scale, d(dO, a, b, h) if dO is not None else None,
                        d(O, a, b, h) if O is not None else None)
            t = bounds(r, e, D, b - a, dtype, grad_dtype)
            for n in names:
                if n == "LSE":
                    got[n][h, a:b], tol[n][h, a:b] = r[n], t[n]
                elif n in ("O", "dQ"):
                    got[n][a:b, h], tol[n][a:b, h] = r[n], t[n]
                else:
                    got[n][a:b, hk] += r[n]
                    tol[n][a:b, hk] += t[n]
    return got, tol


def check(name, x, want, tol):
    """|x - want| <= tol where want is a number; elsewhere (rows of no sequence) nothing is said."""
    x, here = x.double(), ~want.isnan()
    off = torch.where(here, (x - want).abs(), 0.0)
    off = torch.where(here & (x == want), 0.0, off)  # infinities
    bad = ~(off <= torch.where(here, tol, 0.0))
    assert not bad.any(), f"{name}: {int(bad.sum())} values out of bounds, worst {float((off / tol.clamp(min=1e-300))[here].max()):.3g} times"


# ---- the paged cache ------------------------------------------------------------------------------------------------------
def e4m3(x):
    """The nearest e4m3 value, ties to even, of |x| <= 448 (64-bit)."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def least_scale(amax):
    e = math.ceil(math.log2(amax / 448.0)) if amax > 0 else -100
    return 2.0 ** max(e, -100)


def append(k, v, ks, vs, K, V, cu, lens, table, page):
    """The cache (values in 64 bits as [pages, Hkv, page, D] and [pages, Hkv, D, page], scales [pages, Hkv]) with the new tokens, in place."""
    cols = table.shape[1]
    for s in range(len(lens)):
        n, L = cu[s + 1] - cu[s], max(lens[s], 0)
        for col in range(cols):
            a, b = max(L - n, col * page, 0), min(L, (col + 1) * page)
            pid = int(table[s, col])
            if a >= b or not 0 <= pid < k.shape[0]:
                continue
            lo, hi, row = a - col * page, b - col * page, cu[s] + a - (L - n)
            for cache, scales, X in ((k, ks, K), (v.transpose(2, 3), vs, V)):
                x = X[row:row + b - a].double().transpose(0, 1)
                x = torch.where(x.isfinite(), x, math.nan)
                for h in range(x.shape[0]):
                    old = float(scales[pid, h]) if lo else 0.0
                    new = max(least_scale(float(x[h].abs().nan_to_num(0.0).max())), old)
                    cache[pid, h, :lo] = e4m3(cache[pid, h, :lo] * (old / new))
                    cache[pid, h, lo:hi] = e4m3(x[h] / new)
                    scales[pid, h] = new


def cached(Q, cu, lens, table, k, v, ks, vs, page, scale):
    """Attention of the new tokens to the cache (values as above), and bounds."""
    T, Hq, D = Q.shape
    pages, Hkv = ks.shape
    G = Hq // Hkv
    got = {"O": torch.full((T, Hq, D), math.nan, dtype=torch.float64, device=Q.device),
           "LSE": torch.full((Hq, T), math.nan, dtype=torch.float64, device=Q.device)}
    tol = {n: x.clone() for n, x in got.items()}
    for s in range(len(lens)):
        a, b = cu[s], cu[s + 1]
        if a >= b:
            continue
        L = max(lens[s], 0)
        first = L - (b - a)
        pos = [x for x in range(min(L, table.shape[1] * page)) if 0 <= int(table[s, x // page]) < pages]
        idx = torch.tensor(pos, dtype=torch.long, device=Q.device)
        pid, place = table[s].long()[idx // page] if pos else idx, idx % page
        for h in range(Hq):
            hk = h // G
            kk = k[pid, hk, place] * ks[pid, hk].double()[:, None]
            vv = v[pid, hk, :, place] * vs[pid, hk].double()[:, None]
            if len(pos) == min(L, table.shape[1] * page):   # no page is missing: positions are places in the list
                parts = [(torch.arange(b - a), kk, vv, first)]
            else:                                          # else row by row, with the keys that it sees
                parts = [(torch.tensor([i]), kk[idx <= first + i], vv[idx <= first + i], 1 << 30) for i in range(b - a)]
            for rows, k_, v_, f in parts:
                r, e = head(Q[a:b, h].double()[rows.to(Q.device)], k_, v_, f, scale)
                t = bounds(r, e, D, max(1, len(pos)), Q.dtype)
                got["O"][a + rows.to(Q.device), h], got["LSE"][h, a + rows.to(Q.device)] = r["O"], r["LSE"]
                tol["O"][a + rows.to(Q.device), h], tol["LSE"][h, a + rows.to(Q.device)] = t["O"], t["LSE"]
    return got, tol
