"""The gated delta rule token by token in 64 bits, its gradients by the reverse recurrence, and page tables by lists: what the tests of path_delta_* and path_paged_plan
compare with.  Packed tensors (CPU): q, k [T,H,d], v [T,V,d], beta, log_f [T,V], V = H * group; sequences cu[s] .. cu[s+1]."""
import torch

F64 = torch.float64


def batch(lengths, H=2, G=1, d=64, dtype="bf16", gates=True, seed=0, gate_mean=2.0, tail=0):
    """Inputs as the operator meets them: unit q and k, values of size one, beta in (0, 1), gates of a few per cent to a half; `tail` rows behind the last sequence."""
    g = torch.Generator().manual_seed(seed)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    T, V = sum(lengths) + tail, H * G
    rn = lambda *s: torch.randn(*s, generator=g)
    unit = lambda x: torch.nn.functional.normalize(x, dim=-1)
    cu = torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], dtype=torch.int32)
    return dict(q=unit(rn(T, H, d)).to(td), k=unit(rn(T, H, d)).to(td), v=rn(T, V, d).to(td), beta=torch.sigmoid(rn(T, V)).to(td),
                log_f=torch.nn.functional.logsigmoid(rn(T, V) + gate_mean).to(td) if gates else None, cu=cu, d_o=rn(T, V, d).to(td),
                state=0.3 * rn(len(lengths), V, d, d), d_state=rn(len(lengths), V, d, d))


def forward(x, scale, state=None, keep=None):
    """o [T,V,d] (NaN where no sequence has a row) and the last states [nseq,V,d,d]; state: the first ones (None: zeros)."""
    q, k, v, beta = (x[n].to(F64) for n in ("q", "k", "v", "beta"))
    G = v.shape[1] // q.shape[1]
    f = torch.exp(x["log_f"].to(F64)) if x["log_f"] is not None else torch.ones_like(beta)
    cu = x["cu"].tolist()
    o = torch.full(v.shape, float("nan"), dtype=F64)
    last = []
    for s in range(len(cu) - 1):
        S = state[s].to(F64).clone() if state is not None else torch.zeros(v.shape[1], v.shape[2], v.shape[2], dtype=F64)
        for t in range(cu[s], cu[s + 1]):
            kt, qt = k[t].repeat_interleave(G, 0), q[t].repeat_interleave(G, 0)
            if keep is not None:
                keep.append(S.clone())
            S = S * f[t, :, None, None]
            u = beta[t, :, None] * (v[t] - torch.einsum("hij,hi->hj", S, kt))
            S = S + kt[:, :, None] * u[:, None]
            o[t] = scale * torch.einsum("hij,hi->hj", S, qt)
        last.append(S)
    return o, torch.stack(last)


def backward(x, scale, state=None, d_state=None):
    """dq, dk, dv, dbeta, dlog_f, d_state of sum(d_o * o) + sum(d_state * last states)."""
    q, k, v, beta, d_o = (x[n].to(F64) for n in ("q", "k", "v", "beta", "d_o"))
    H, G = q.shape[1], v.shape[1] // q.shape[1]
    f = torch.exp(x["log_f"].to(F64)) if x["log_f"] is not None else torch.ones_like(beta)
    kept = []
    _, last = forward(x, scale, state, kept)
    cu = x["cu"].tolist()
    dq, dk, dv, db, dl = (torch.zeros(*a.shape, dtype=F64) for a in (q, k, v, beta, beta))
    first = torch.zeros_like(last)
    fold = lambda a: a.view(H, G, -1).sum(1)
    for s in range(len(cu) - 1):
        g = d_state[s].to(F64).clone() if d_state is not None else torch.zeros_like(last[s])
        for t in range(cu[s + 1] - 1, cu[s] - 1, -1):
            kt, qt = k[t].repeat_interleave(G, 0), q[t].repeat_interleave(G, 0)
            old = kept[t - cu[0]] * f[t, :, None, None]
            e = v[t] - torch.einsum("hij,hi->hj", old, kt)
            u = beta[t, :, None] * e
            new = old + kt[:, :, None] * u[:, None]
            dq[t] = fold(scale * torch.einsum("hij,hj->hi", new, d_o[t]))
            g = g + scale * qt[:, :, None] * d_o[t][:, None]
            du = torch.einsum("hij,hi->hj", g, kt)
            db[t] = (du * e).sum(-1)
            dv[t] = beta[t, :, None] * du
            dk[t] = fold(torch.einsum("hij,hj->hi", g, u) - torch.einsum("hij,hj->hi", old, dv[t]))
            g = g - kt[:, :, None] * dv[t][:, None]
            dl[t] = (g * old).sum((-1, -2))
            g = g * f[t, :, None, None]
        first[s] = g
    return dq, dk, dv, db, dl, first


def plan(cached, new, table, free, count, T, page):
    """path_paged_plan on lists: table [nseq][pages_per_seq], free [num_pages], count an int.  Returns (table, free, count, cu, slots, missing)."""
    pool, P = len(free), len(table[0])
    table, free, count = [list(r) for r in table], list(free), min(max(count, 0), pool)
    ok = lambda e: 0 <= e < pool
    cached = [max(c, 0) for c in cached]
    cu = [0]
    for m in new:
        cu.append(min(cu[-1] + max(m, 0), T))
    # (an offset ends at T; what is behind it counts for nothing)
    n = [cu[s + 1] - cu[s] for s in range(len(new))]
    want = [min(P, -(-(c + m) // page)) for c, m in zip(cached, n)]
    have = [-(-c // page) for c in cached]
    for s, row in enumerate(table):
        for j in range(want[s], P):
            if ok(row[j]) and count < pool:
                free[count] = row[j]
                count += 1
            row[j] = -1
    missing = [0] * len(table)
    for s, row in enumerate(table):
        for j in range(have[s], want[s]):
            if not ok(row[j]):
                if count > 0:
                    count -= 1
                    row[j] = free[count]
                else:
                    row[j] = -1
                    missing[s] += 1
    slots = [-1] * T
    for s, row in enumerate(table):
        for t in range(cu[s], cu[s + 1]):
            j, i = divmod(cached[s] + t - cu[s], page)
            if j < P and ok(row[j]):
                slots[t] = row[j] * page + i
    return table, free, count, cu, slots, missing
