"""Serving from a paged cache: attention of new tokens over it, appending them to it, and both in one call.

PaTH attention's logit of query i and key j is ``scale q_i^T H_i .. H_{j+1} k_j``, ``H_t = I - beta_t w_t w_t^T``.  A paged
cache holds, of n tokens, the keys carried to the last one, ``H_{n-1} .. H_{i+1} k_i``, and the values, in pages of a pool
[num_pages, H, page, d]; with forget gates also the running sums of their logarithms.  Operators (``op`` of a case):

  attn    o and lse of m new tokens over the n cached ones and over each other; the cache is only read
  append  the cached keys carried on by the new tokens' transitions, the new keys and values written behind them
  extend  both in one call

``listed()`` names the cases, ``draw()`` gives further ones of the same ranges, ``prepare()`` makes what a server holds before
the call, ``run()`` is one call (``own``) or the same in elementary operations in 32 bits, ``exact()`` the definition token by
token in 64 bits, ``work()`` the bytes and operations that a call cannot do without.
"""
from __future__ import annotations

import math
import random

import torch

own = False

MAX_CACHE = 32 * 16 * 8192 * 128            # cached key elements of a drawn case
MAX_PAIRS = 16 * 2048 * 20000 * 128         # query-key pairs of a drawn case, times d


def _case(op, S, H, cached, new, d=128, group=1, page=64, dtype="bf16", gates=False, shortest=None, spread="same"):
    return dict(op=op, S=S, H=H, group=group, cached=cached, shortest=cached if shortest is None else shortest, new=new,
                spread=spread, d=d, page=page, dtype=dtype, gates=gates)


def listed():
    return [
        # a decoding batch looking at its cache (the appends of several tokens deferred): bound by memory
        dict(name="attn_token_32x8192", **_case("attn", 32, 16, 8192, 1)),
        # drafted tokens being verified, heads sharing keys, sequences of all lengths, small pages
        dict(name="attn_drafts_16x4000_group4", **_case("attn", 16, 8, 4000, 6, group=4, page=16, shortest=300, spread="ragged")),
        # a chunk of a long prompt
        dict(name="attn_chunk_512_over_8192", **_case("attn", 1, 16, 8192, 512)),
        # a batch as a server runs it: one chunk of a prompt, everybody else one token; gates, narrow heads, odd lengths
        dict(name="attn_mixed_12x3001_d64_gates", **_case("attn", 12, 16, 3001, 700, d=64, gates=True, shortest=77, spread="one_long")),
        # a small fp32 chunk, as a check of a model's port runs it
        dict(name="attn_chunk_100_over_300_d64_fp32", **_case("attn", 2, 2, 300, 100, d=64, dtype="fp32", page=16)),
        # accepted drafts appended
        dict(name="append_drafts_16x4000", **_case("append", 16, 16, 4000, 4, page=16, shortest=300, spread="ragged")),
        # a chunk appended to a long cache
        dict(name="append_chunk_512_over_8192", **_case("append", 1, 16, 8192, 512)),
        # one sequence early in its decoding: latency
        dict(name="extend_token_1x500", **_case("extend", 1, 16, 500, 1)),
        # a decoding batch with gates, narrow heads, odd lengths
        dict(name="extend_token_8x3001_d64_gates", **_case("extend", 8, 16, 3001, 1, d=64, gates=True, shortest=1500, spread="ragged")),
        # a decoding batch over long caches: bound by memory
        dict(name="extend_token_32x8192", **_case("extend", 32, 16, 8192, 1)),
        # the first chunk of a prompt: nothing cached yet
        dict(name="extend_chunk_1000_over_0", **_case("extend", 1, 16, 0, 1000)),
        # a large chunk over a long context, heads in pairs; the largest
        dict(name="extend_chunk_2048_over_16384_group2", **_case("extend", 1, 8, 16384, 2048, group=2, page=128)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: one token, a few drafts, or a chunk, over nothing up to a long cache (lengths on a logarithmic scale, odd
    ones among them), with as many sequences as the bounds on cache and pairs leave room for."""
    op = rng.choice(["attn", "append", "extend"])
    kind = rng.choice(["token", "drafts", "chunk", "chunk", "mixed"])
    d = rng.choice([64, 128])
    dtype = "fp32" if rng.random() < 0.15 else "bf16"
    H = rng.choice([1, 2, 4]) if dtype == "fp32" else rng.choice([2, 4, 8, 16, 32])
    group = rng.choice([1, 1, 1, 2, 4, 8]) if H <= 8 else 1
    top = 2000 if dtype == "fp32" else 32768
    cached = 0 if kind != "token" and rng.random() < 0.12 else _log_int(rng, 8, top)
    new = {"token": 1, "drafts": rng.randint(2, 16)}.get(kind) or _log_int(rng, 17, min(2048, top // 4))
    while new > 1 and H * group * new * (cached + new) * d > MAX_PAIRS:
        new = new // 2 + 1
    most = max(1, min(64, MAX_CACHE // (H * (cached + new) * d), MAX_PAIRS // (H * group * new * (cached + new) * d)))
    if kind in ("chunk", "mixed"):
        most = min(most, 12 if kind == "mixed" else 4, max(1, 24000 // (H * group * new)))      # (the plain form pads every sequence to the longest chunk)
    S = _log_int(rng, 1, most) if most > 1 else 1
    return _case(op, S, H, cached, new, d=d, group=group, page=rng.choice([16, 32, 64, 128, 256]), dtype=dtype, gates=rng.random() < 0.3,
                 shortest=rng.choice([cached, max(0, cached // 10)]), spread="one_long" if kind == "mixed" else rng.choice(["same", "ragged"]) if new > 1 else "same")


def _lengths(case):
    """Cached and new tokens of each sequence: between the shortest and the longest (which occurs), in no order; new tokens all
    alike, spread from one up, or one chunk among single tokens."""
    S, rng = case["S"], random.Random(f"{case['S']} {case['shortest']} {case['cached']} {case['new']}")
    old = [rng.randint(case["shortest"], case["cached"]) for _ in range(S)]
    old[S // 2] = case["cached"]
    new = [case["new"]] * S
    if case["spread"] == "ragged":
        new = [rng.randint(1, case["new"]) for _ in range(S)]
    elif case["spread"] == "one_long":
        new = [1] * S
    new[S // 3] = case["new"]
    return old, new


def prepare(case, seed):
    S, H, G, d, page = case["S"], case["H"], case["group"], case["d"], case["page"]
    dev = torch.device("cuda")
    td = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *shape: torch.randn(*shape, device=dev, generator=gen)
    old, new = _lengths(case)
    per = max(-(-(a + b) // page) for a, b in zip(old, new))
    pool = S * per + 3                                         # a few pages belong to nobody
    order = torch.randperm(pool, device=dev, generator=gen)[:S * per]      # pages lie anywhere
    T = sum(new)
    s = dict(case=case, scale=d ** -0.5, T=T, max_new=max(new), max_cached=max(old),
             page_table=order.view(S, per).to(torch.int32).contiguous(),
             cached=torch.tensor(old, dtype=torch.int32, device=dev),
             cu_new=torch.tensor([0] + [sum(new[:i + 1]) for i in range(S)], dtype=torch.int32, device=dev),
             kpages=rn(pool, H, page, d).to(td), vpages=rn(pool, H, page, d).to(td),
             k=rn(T, H, d).to(td), v=rn(T, H, d).to(td), w=torch.nn.functional.normalize(rn(T, H, d), dim=-1).to(td),
             beta=(2 * torch.sigmoid(rn(T, H))).to(td), q=rn(T, H * G, d).to(td), log_f=None, cpages=None, ws=None)
    if case["gates"]:      # gates of a few per cent a token; their sums along each sequence
        s["log_f"] = torch.nn.functional.logsigmoid(rn(T, H) + 3.0).to(td)
        c = torch.cumsum(torch.nn.functional.logsigmoid(rn(S, H, per * page) + 3.0), -1)
        s["cpages"] = torch.zeros(pool, H, page, device=dev)
        s["cpages"][order] = c.view(S, H, per, page).transpose(1, 2).reshape(S * per, H, page)
    if own:      # the scratch memory that a server keeps
        import paper_2505_16381_amd as pa
        dt = pa.PATH_BF16 if case["dtype"] == "bf16" else pa.PATH_F32
        s["ws"] = torch.empty(pa.path_paged_workspace_bytes(S, T, s["max_new"], s["max_cached"], H, G, d, dt), dtype=torch.uint8, device=dev)
    return s


def run(s):
    if not own:
        return _plain(s)
    import paper_2505_16381_amd as pa
    op = s["case"]["op"]
    more = dict(log_f=s["log_f"], cpages=s["cpages"], workspace=s["ws"])
    cache = (s["kpages"], s["vpages"], s["page_table"], s["cached"], s["cu_new"], s["max_new"], s["max_cached"])
    kvwb = (s["k"], s["v"], s["w"], s["beta"])
    if op == "append":
        pa.path_paged_append(*kvwb, *cache, **more)
        return _pages(s)
    call = pa.path_paged_attn if op == "attn" else pa.path_paged_extend
    o, lse = call(s["q"], *kvwb, *cache, scale=s["scale"], **more)
    return (o, lse) if op == "attn" else (o, lse, *_pages(s))


def _pages(s):
    return (s["kpages"], s["vpages"]) if s["cpages"] is None else (s["kpages"], s["vpages"], s["cpages"])


# ---- the plain form -------------------------------------------------------------------------------------------------

def _block_inverses(N, size):
    """Inverses of the size x size diagonal blocks of I + N, N strictly lower triangular, from those of half the size."""
    M = N.shape[-1]
    if size == 1:
        return torch.ones(*N.shape[:-2], M, 1, 1, dtype=N.dtype, device=N.device)
    half = size // 2
    inv = _block_inverses(N, half)
    top, bottom = inv[..., 0::2, :, :], inv[..., 1::2, :, :]
    at = torch.arange(M // size, device=N.device)
    below = N.unflatten(-2, (M // size, size)).unflatten(-1, (M // size, size))[..., at, half:, at, :half].movedim(0, -3)
    left = torch.cat([top, -(bottom @ below @ top)], -2)
    right = torch.cat([torch.zeros_like(top), bottom], -2)
    return torch.cat([left, right], -1)


def _plain(s):
    """Every sequence padded to the longest chunk (beta = 0, w = 0 behind its end) and to the longest cache."""
    case, op = s["case"], s["case"]["op"]
    S, H, G, d = case["S"], case["H"], case["group"], case["d"]
    dev = s["k"].device
    new = (s["cu_new"][1:] - s["cu_new"][:-1]).long()
    M = s["max_new"]
    a = torch.arange(M, device=dev)
    there = a < new[:, None]                                                           # [S, M]
    at = (s["cu_new"][:-1, None].long() + a).clamp(max=s["T"] - 1)
    take = lambda x: (x[at].float() * there.view(S, M, *[1] * (x.dim() - 1))).transpose(1, 2)       # [S, heads, M, ..]
    k, v, w, beta = take(s["k"]), take(s["v"]), take(s["w"]), take(s["beta"])
    table = s["page_table"].long()
    cached = s["cached"].long()
    n = s["max_cached"]
    row = torch.arange(n, device=dev)
    flat = lambda pages: pages[table].transpose(1, 2).flatten(2, 3)[:, :, :n].float()              # [S, H, n, ..]
    K = flat(s["kpages"])
    seen = row < cached[:, None]                                                       # [S, n]
    # the triangular transform of the chunk
    A = torch.tril(w @ w.mT, -1)
    size = 1 << max(0, M - 1).bit_length()
    N = torch.nn.functional.pad(beta[..., None] * A, (0, size - M, 0, size - M))
    Tm = _block_inverses(N, size)[..., 0, :M, :M] * beta[..., None, :]
    D = torch.tril(w @ k.mT, -1)
    if s["log_f"] is not None:
        C = flat(s["cpages"][..., None])[..., 0]                                        # [S, H, n]
        start = torch.where(cached > 0, 1.0, 0.0)[:, None] * C.gather(2, (cached - 1).clamp(min=0)[:, None, None].expand(S, H, 1))[..., 0] if n else torch.zeros(S, H, device=dev)
        c = start[..., None] + torch.cumsum(take(s["log_f"]), -1)                       # [S, H, M]
    out = ()
    if op != "append":
        q = take(s["q"]).unflatten(1, (H, G))                                           # [S, H, G, M, d]
        L = torch.tril(q @ w.mT[:, :, None])
        LT = L @ Tm[:, :, None]
        inner = (q @ k.mT[:, :, None] - LT @ D[:, :, None]) * s["scale"]
        outer = (q - LT @ w[:, :, None]) @ K.mT[:, :, None] * s["scale"]
        if s["log_f"] is not None:
            inner = inner + (c[..., :, None] - c[..., None, :])[:, :, None]
            outer = outer + (c[..., :, None] - C[..., None, :])[:, :, None]
        inner = inner.masked_fill(a[:, None] < a, -math.inf)
        outer = outer.masked_fill(~seen[:, None, None, None], -math.inf)
        top = inner.amax(-1) if n == 0 else torch.maximum(inner.amax(-1), outer.amax(-1))
        inner, outer = torch.exp(inner - top[..., None]), torch.exp(outer - top[..., None])
        total = inner.sum(-1) + outer.sum(-1)
        V = flat(s["vpages"]).masked_fill(~seen[:, None, :, None], 0.0)
        o = (inner @ v[:, :, None] + outer @ V[:, :, None]) / total[..., None]
        lse = top + torch.log(total)
        o, lse = o.flatten(1, 2).transpose(1, 2), lse.flatten(1, 2).transpose(1, 2)      # [S, M, heads, ..]
        out = (o[there].to(s["q"].dtype), lse[there])
    if op == "attn":
        return out
    # the cached keys carried on, the new ones carried to the chunk's end
    K = K - (K @ (Tm @ w).mT) @ w
    k = k - (Tm @ D).mT @ w
    which, pos = seen.nonzero(as_tuple=True)
    size = case["page"]
    s["kpages"][table[which, pos // size], :, pos % size] = K.transpose(1, 2)[which, pos].to(s["kpages"].dtype)
    which, tok = there.nonzero(as_tuple=True)
    pos = cached[which] + tok
    page, slot = table[which, pos // size], pos % size
    s["kpages"][page, :, slot] = k.transpose(1, 2)[which, tok].to(s["kpages"].dtype)
    s["vpages"][page, :, slot] = s["v"]
    if s["log_f"] is not None:
        s["cpages"][page, :, slot] = c.transpose(1, 2)[which, tok]
    return (*out, *_pages(s))


# ---- the definition, token by token, in 64 bits -----------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op, S, H, G, page = case["op"], case["S"], case["H"], case["group"], case["page"]
    old, new = _lengths(case)
    if sum(m * H * (G * m * (op != "append") + n * (op != "attn")) for n, m in zip(old, new)) * case["d"] * 8 > 12e12:
        return None
    o, lse = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    kp, vp = (s["kpages"].double(), s["vpages"].double()) if op != "attn" else (None, None)
    cp = s["cpages"].double() if s["cpages"] is not None else None
    first = 0
    for i, (n, m) in enumerate(zip(old, new)):
        mine = slice(first, first + m)
        first += m
        pos = torch.arange(n + m, device="cuda")
        at, slot = s["page_table"][i].long()[pos // page], pos % page
        K, V = (s[x][at[:n], :, slot[:n]].double().transpose(0, 1) for x in ("kpages", "vpages"))       # [H, n, d]
        k, v, w, b = (s[x][mine].double().transpose(0, 1) for x in ("k", "v", "w", "beta"))
        if cp is not None:
            start = cp[at[n - 1], :, slot[n - 1]] if n else torch.zeros(H, dtype=torch.float64, device="cuda")
            c = start[:, None] + torch.cumsum(s["log_f"][mine].double().T, -1)                          # [H, m]
            C = cp[at[:n], :, slot[:n]].T
        if op != "append":
            # every query walks left: the logit with a token's key, then that token's transition
            x = s["q"][mine].double().view(m, H, G, -1).permute(1, 2, 0, 3).contiguous()                # [H, G, m, d]
            z = torch.full((H, G, m, n + m), -math.inf, dtype=torch.float64, device="cuda")
            for t in range(m - 1, -1, -1):
                y = x[:, :, t:]
                z[:, :, t:, n + t] = (y * k[:, None, None, t]).sum(-1)
                y -= b[:, None, None, t, None] * (y * w[:, None, None, t]).sum(-1, keepdim=True) * w[:, None, None, t]
            z[..., :n] = torch.matmul(x.flatten(1, 2), K.mT.contiguous()).view(H, G, m, n)
            z *= s["scale"]
            if cp is not None:
                z += (c[:, :, None] - torch.cat([C, c], -1)[:, None])[:, None]
            top = z.amax(-1, keepdim=True)
            z = torch.exp(z - top)
            total = z.sum(-1, keepdim=True)
            y = torch.matmul(z.flatten(1, 2), torch.cat([V, v], 1)).view(H, G, m, -1) / total
            o[mine] = y.permute(2, 0, 1, 3).flatten(1, 2)
            lse[mine] = (top + torch.log(total))[..., 0].permute(2, 0, 1).flatten(1, 2)
            del z
        if op != "attn":
            K = torch.cat([K, k], 1)
            for t in range(m):      # a token arrives: the keys before it take its transition
                y = K[:, :n + t]
                y -= b[:, t, None, None] * (y * w[:, t, None]).sum(-1, keepdim=True) * w[:, t, None]
            kp[at, :, slot] = K.transpose(0, 1)
            vp[at[n:], :, slot[n:]] = v.transpose(0, 1)
            if cp is not None:
                cp[at[n:], :, slot[n:]] = c.T
    out = (o, lse) if op != "append" else ()
    if op != "attn":
        out += (kp, vp) if cp is None else (kp, vp, cp)
    return out


def work(case):
    """Each cached key and value that is needed read once, each carried key written once, the new tokens read, the results
    written; 4 d operations per query and key it attends to, 4 d per cached key and (up to d / 2) new token for the transitions."""
    op, H, G, d = case["op"], case["H"], case["group"], case["d"]
    es, g = (2 if case["dtype"] == "bf16" else 4), (1 if case["gates"] else 0)
    old, new = _lengths(case)
    n, T = sum(old), sum(new)
    nbytes, flops = T * H * (3 * d + 1 + g) * es, 0.0
    if op != "append":
        nbytes += n * H * (2 * d * es + 4 * g) + T * H * G * (2 * d * es + 4)
        flops += 4.0 * d * H * G * sum(b * a + b * (b + 1) / 2 for a, b in zip(old, new))
    if op != "attn":
        nbytes += n * H * d * es * (2 if op == "append" else 1) + T * H * (2 * d * es + 4 * g)
        flops += 4.0 * d * H * sum(min(b, d // 2) * a for a, b in zip(old, new))
    return {"bytes": float(nbytes), "flops": flops}
