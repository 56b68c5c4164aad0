"""Paged caches in 64 bits on the CPU: random batches, and what attention over them and appends to them leave (plain torch, token by
token from the definition; nothing of the library)."""
import math

import torch


def batch(old, new, H, G, d, page, dtype, gates=False, seed=0, spare=2, beta=None, unused=math.nan):
    """A batch of sequences with `old` cached and `new` new tokens, its pages in random order; every slot that holds no token
    is `unused`."""
    gen = torch.Generator().manual_seed(seed)
    td = torch.float32 if dtype == "fp32" else torch.bfloat16
    rn = lambda *shape: torch.randn(*shape, generator=gen)
    S, T = len(old), sum(new)
    per = max(1, max(-(-(a + b) // page) for a, b in zip(old, new)))
    pool = S * per + spare
    table = torch.randperm(pool, generator=gen)[:S * per].view(S, per).to(torch.int32)
    x = dict(q=rn(T, H * G, d), k=rn(T, H, d), v=rn(T, H, d), w=torch.nn.functional.normalize(rn(T, H, d), dim=-1),
             beta=2 * torch.sigmoid(rn(T, H)) if beta is None else torch.full((T, H), float(beta)))
    x = {n: t.to(td) for n, t in x.items()}
    x["log_f"] = torch.nn.functional.logsigmoid(rn(T, H) + 2).to(td) if gates else None
    x["kpages"] = torch.full((pool, H, page, d), unused, dtype=td)
    x["vpages"] = torch.full((pool, H, page, d), unused, dtype=td)
    x["cpages"] = torch.full((pool, H, page), unused) if gates else None
    for s, n in enumerate(old):
        c = torch.cumsum(torch.nn.functional.logsigmoid(rn(H, n) + 2), -1)
        for i in range(0, n, page):
            b = min(page, n - i)
            p = int(table[s, i // page])
            x["kpages"][p, :, :b] = rn(H, b, d).to(td)
            x["vpages"][p, :, :b] = rn(H, b, d).to(td)
            if gates:
                x["cpages"][p, :, :b] = c[:, i:i + b]
    x.update(page_table=table, cached=torch.tensor(old, dtype=torch.int32),
             cu_new=torch.tensor([0] + [sum(new[:i + 1]) for i in range(S)], dtype=torch.int32))
    return x


def rows_of(x, s, n):
    """(pages, slots) of the first n tokens of sequence s; pages outside the pool are -1."""
    page = x["kpages"].shape[2]
    pos = torch.arange(n)
    p = x["page_table"][s].long()[pos // page] if n else pos
    return torch.where((p >= 0) & (p < x["kpages"].shape[0]), p, torch.tensor(-1)), pos % page


def expect(x, scale, op):
    """(o, lse, kpages, vpages, cpages) after attn / append / extend, in 64 bits; rows and slots that are not written: NaN in o and
    lse, as they were in the pages."""
    T, H, d = x["k"].shape
    G = x["q"].shape[1] // H
    o, lse = torch.full((T, H * G, d), math.nan, dtype=torch.float64), torch.full((T, H * G), math.nan, dtype=torch.float64)
    kp, vp = x["kpages"].double().clone(), x["vpages"].double().clone()
    cp = x["cpages"].double().clone() if x["cpages"] is not None else None
    cu = x["cu_new"].tolist()
    for s, n in enumerate(x["cached"].tolist()):
        t0, m = cu[s], cu[s + 1] - cu[s]
        pages, slots = rows_of(x, s, n)
        here = pages >= 0
        pages, slots = pages[here], slots[here]
        K, V = kp[pages, :, slots].transpose(0, 1), x["vpages"].double()[pages, :, slots].transpose(0, 1)      # [H, n, d]
        k, v, w, b = (x[i][t0:t0 + m].double().transpose(0, 1) for i in ("k", "v", "w", "beta"))
        if cp is not None:
            lp, ls = rows_of(x, s, n)
            start = cp[lp[-1], :, ls[-1]] if n and lp[-1] >= 0 else torch.zeros(H, dtype=torch.float64)
            c = start[:, None] + torch.cumsum(x["log_f"][t0:t0 + m].double().T, -1)
            C = cp[pages, :, slots].T
        if op != "append":
            for a in range(m):
                u = x["q"][t0 + a].double().view(H, G, d).clone()
                z = torch.empty(H, G, a + 1, dtype=torch.float64)
                for t in range(a, -1, -1):
                    z[..., t] = (u * k[:, None, t]).sum(-1)
                    u -= b[:, t, None, None] * (u * w[:, None, t]).sum(-1, keepdim=True) * w[:, None, t]
                z = torch.cat([u @ K.mT, z], -1) * scale
                if cp is not None:
                    z += (c[:, a, None] - torch.cat([C, c[:, :a + 1]], -1))[:, None]
                p = torch.softmax(z, -1)
                o[t0 + a] = (p @ torch.cat([V, v[:, :a + 1]], 1)).reshape(H * G, d)
                lse[t0 + a] = torch.logsumexp(z, -1).reshape(-1)
        if op != "attn" and m:
            K = torch.cat([K, k], 1)
            old = K.shape[1] - m
            for t in range(m):
                y = K[:, :old + t]
                y -= b[:, t, None, None] * (y * w[:, None, t]).sum(-1, keepdim=True) * w[:, None, t]
            kp[pages, :, slots] = K[:, :old].transpose(0, 1)
            page, per = x["kpages"].shape[2], x["page_table"].shape[1]
            for t in range(m):
                i = n + t
                if i // page >= per or not 0 <= int(x["page_table"][s, i // page]) < kp.shape[0]:
                    continue
                at = int(x["page_table"][s, i // page])
                kp[at, :, i % page] = K[:, old + t]
                vp[at, :, i % page] = v[:, t]
                if cp is not None:
                    cp[at, :, i % page] = c[:, t]
    return o, lse, kp, vp, cp


def drop_pages(x, holes, num_pages):
    """The batch with table entries at (sequence, page) in `holes` pointing outside the pool."""
    for i, (s, p) in enumerate(holes):
        x["page_table"][s, p] = (-1, num_pages, num_pages + 12345, -2 ** 31)[i % 4]
    return x
