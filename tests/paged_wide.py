"""Paged caches in 64 bits for batches too wide for paged_model.py (same definition, token by token, all queries and heads at once; on any device), and the bars that
the documented accuracy gives.

Bars.  Inputs are standard normal (q, k, v), w of length one, scale d^-1/2.
  A number kept as a pair of bf16 numbers is off by r = 2.6e-6 of itself, in the mean: the first one's rest is 2^-7 / sqrt(12) of the binade, the second one's as much of
  that (2.26e-3 squared, and half of it lost to where in its binade a number lies).  fp32 matrix products of 64 to 128 terms: r = 2^-24 sqrt(128) / 2 = 3.4e-7.
  A row's x, or a key, that went through N such roundings is off by at most 2 r sqrt(N) sqrt(d) in length (each is of a vector at most twice as long), in no
  direction of its own: a logit by 2 r sqrt(N), and so is each element of a key.  Few tokens: x itself, N = 1.  Chunks: five for forming x in its tile (L, T, their
  product's parts, x), five for each of t tiles that it crosses, six for the keys' side: N = 5 (t + 1) + 6.
  lse   six deviations, 12 r sqrt(N), and 1e-5 for fp32 sums and the hardware's exp and log; with gates 5e-7 of the largest |c| (eight roundings of it).
  keys  bf16: the result is rounded once, 2^-8 |k'|, and 12 r sqrt(N).  Cached keys of a chunk: the matrix's elements are fp16 numbers, off by
        2^-10 / sqrt(12) * 0.72 = 2e-4 of themselves, rows of length at most 2 meet keys whose elements are about 1.2: six deviations are 2.9e-3 more.
  o     bf16: each weight is rounded once, 2^-8 of the mean of |v| over the weights, the result once, 2^-8 |o|; weights are off by the lse's bar, twice.
        fp32: that last term and 1e-5.
A part lost anywhere makes its r 1.6e-3, six hundred times as large."""
import math

import torch

PAIR, SUM32, HALF = 2.6e-6, 3.4e-7, 2.9e-3


def batch(old, new, H, G, d, page, dtype, gates=False, seed=0, device="cuda"):
    gen = torch.Generator(device=device).manual_seed(seed)
    td = torch.float32 if dtype == "fp32" else torch.bfloat16
    rn = lambda *shape: torch.randn(*shape, generator=gen, device=device)
    S, T = len(old), sum(new)
    per = max(-(-(a + b) // page) for a, b in zip(old, new))
    pool = S * per + 2
    table = torch.randperm(pool, generator=gen, device=device)[:S * per].view(S, per).to(torch.int32)
    x = dict(q=rn(T, H * G, d).to(td), k=rn(T, H, d).to(td), v=rn(T, H, d).to(td), w=torch.nn.functional.normalize(rn(T, H, d), dim=-1).to(td),
             beta=(2 * torch.sigmoid(rn(T, H))).to(td), log_f=torch.nn.functional.logsigmoid(rn(T, H) + 2).to(td) if gates else None)
    nan = lambda *shape, dtype=td: torch.full(shape, math.nan, dtype=dtype, device=device)
    x.update(kpages=nan(pool, H, page, d), vpages=nan(pool, H, page, d), cpages=nan(pool, H, page, dtype=torch.float32) if gates else None)
    for s, n in enumerate(old):
        c = torch.cumsum(torch.nn.functional.logsigmoid(rn(H, n) + 2), -1)
        for i in range(0, n, page):
            b, p = min(page, n - i), int(table[s, i // page])
            x["kpages"][p, :, :b], x["vpages"][p, :, :b] = rn(H, b, d).to(td), rn(H, b, d).to(td)
            if gates:
                x["cpages"][p, :, :b] = c[:, i:i + b]
    x.update(page_table=table, cached=torch.tensor(old, dtype=torch.int32, device=device),
             cu_new=torch.tensor([0] + [sum(new[:i + 1]) for i in range(S)], dtype=torch.int32, device=device))
    return x


def walk(x, s):
    """What sequence s's queries are at the chunk's start, [H, G, m, d], and their logits with the new keys, [H, G, m, m]: from the last token to the
    first, each query's logit with a token's key, then that token's transition."""
    H = x["k"].shape[1]
    cu = x["cu_new"].tolist()
    t0, m = cu[s], cu[s + 1] - cu[s]
    k, w, b = (x[i][t0:t0 + m].double().transpose(0, 1) for i in ("k", "w", "beta"))
    u = x["q"][t0:t0 + m].double().view(m, H, -1, x["q"].shape[2]).permute(1, 2, 0, 3).contiguous()
    z = torch.full((*u.shape[:3], m), -math.inf, dtype=torch.float64, device=u.device)
    for t in range(m - 1, -1, -1):
        y = u[:, :, t:]
        z[:, :, t:, t] = (y * k[:, None, None, t]).sum(-1)
        y -= b[:, None, None, t, None] * (y * w[:, None, None, t]).sum(-1, keepdim=True) * w[:, None, None, t]
    return u, z


def cached(x, s, names):
    page, n = x["kpages"].shape[2], int(x["cached"][s])
    pos = torch.arange(n, device=x["k"].device)
    at = x["page_table"][s].long()[pos // page]
    return [x[i][at, :, pos % page].double().transpose(0, 1).contiguous() for i in names]


def expect(x, scale, op, change=lambda u: u):
    """o, lse, the weights' mean of |v|, and the pages, in 64 bits.  ``change`` is applied to the queries that meet the cached keys."""
    T, H, d = x["k"].shape
    dev, page = x["k"].device, x["kpages"].shape[2]
    o, lse = torch.empty(x["q"].shape, dtype=torch.float64, device=dev), torch.empty(x["q"].shape[:2], dtype=torch.float64, device=dev)
    size = torch.empty_like(o)
    kp, vp, cp = (x[n].clone() if x[n] is not None else None for n in ("kpages", "vpages", "cpages"))
    kp = kp.double()
    cu = x["cu_new"].tolist()
    for s, n in enumerate(x["cached"].tolist()):
        t0, m = cu[s], cu[s + 1] - cu[s]
        if not m:
            continue
        K, V = cached(x, s, ("kpages", "vpages"))
        k, v, w, b = (x[i][t0:t0 + m].double().transpose(0, 1) for i in ("k", "v", "w", "beta"))
        if cp is not None:
            C = cached(x, s, ("cpages",))[0]
            c = (C[:, -1:] if n else 0) + torch.cumsum(x["log_f"][t0:t0 + m].double().T, -1)
        if op != "append":
            u, z = walk(x, s)
            u = change(u)
            G = u.shape[1]
            z = torch.cat([torch.matmul(u.flatten(1, 2), K.mT.contiguous()).view(H, G, m, n), z], -1) * scale
            if cp is not None:
                z += (c[:, :, None] - torch.cat([C, c], -1)[:, None])[:, None]
            top = z.amax(-1, keepdim=True)
            z = torch.exp(z - top)
            total = z.sum(-1, keepdim=True)
            z /= total
            vv = torch.cat([V, v], 1)
            out = lambda y: torch.matmul(z.flatten(1, 2), y).view(H, G, m, d).permute(2, 0, 1, 3).flatten(1, 2)
            o[t0:t0 + m], size[t0:t0 + m] = out(vv), out(vv.abs())
            lse[t0:t0 + m] = (top + torch.log(total))[..., 0].permute(2, 0, 1).flatten(1, 2)
            del z
        if op != "attn":
            K = torch.cat([K, k], 1)
            for t in range(m):
                y = K[:, :n + t]
                y -= b[:, t, None, None] * (y * w[:, t, None]).sum(-1, keepdim=True) * w[:, t, None]
            pos = torch.arange(n + m, device=dev)
            at, slot = x["page_table"][s].long()[pos // page], pos % page
            kp[at, :, slot] = K.transpose(0, 1)
            vp[at[n:], :, slot[n:]] = x["v"][t0:t0 + m]
            if cp is not None:
                cp[at[n:], :, slot[n:]] = c.T.float()
    return o, lse, size, kp, vp, cp


def bars(x, few_limit=16):
    """r, lse's bar, what a key may be off besides its rounding (cached ones of a chunk: HALF more), for the whole batch."""
    G = x["q"].shape[1] // x["k"].shape[1]
    new = (x["cu_new"][1:] - x["cu_new"][:-1])
    most = int(new.max())
    limit = min(few_limit, 64 // G)
    chunk = most > limit or (len(new) == 1 and most > limit)
    r = SUM32 if x["k"].dtype == torch.float32 else PAIR
    N = 5 * ((most - 1) // 64 + 1) + 6 if chunk else 1
    key = 12 * r * math.sqrt(N)
    c = 0.0 if x["cpages"] is None else float(x["cpages"].nan_to_num().abs().max()) + float(x["log_f"].float().abs().sum(0).max())
    return r, key + 1e-5 + 5e-7 * c, key + (1e-6 if r == SUM32 else 0), chunk


def compare(x, y, got, want, op):
    """The call's outputs and pages y against ``want`` (and pages that it leaves against x)."""
    o, lse, size, kp, vp, cp = want
    r, lse_bar, key_bar, chunk = bars(x)
    f32 = r == SUM32
    if op != "append":
        off = (got[1].double() - lse).abs().max()
        assert off <= lse_bar, (float(off), lse_bar)
        vmax = max(float(size.max()), 1.0)
        bar = (1e-5 if f32 else 0) + (0 if f32 else 2 ** -8) * (size + o.abs()) + 2 * lse_bar * vmax
        assert ((got[0].double() - o).abs() <= bar).all(), float(((got[0].double() - o).abs() - bar).max())
    same = lambda a, b: torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    if op == "attn":
        assert same(y["kpages"], x["kpages"]) and same(y["vpages"], x["vpages"])
        return
    assert torch.equal(y["kpages"].isnan(), kp.isnan())
    fresh = x["kpages"].isnan() & ~kp.isnan()      # slots of the new tokens
    off = (y["kpages"].double() - kp).abs() - (0 if f32 else 2 ** -8) * kp.abs()
    assert off[fresh].max() <= key_bar, (float(off[fresh].max()), key_bar)
    old = ~kp.isnan() & ~fresh
    if old.any():
        bar = key_bar + (HALF if chunk and not f32 else 0)
        assert off[old].max() <= bar, (float(off[old].max()), bar)
    assert same(y["vpages"], vp)
    if cp is not None:
        assert torch.equal(y["cpages"].isnan(), cp.isnan())
        assert (y["cpages"] - cp).nan_to_num().abs().max() <= 5e-7 * max(1.0, float(cp.nan_to_num().abs().max()))
