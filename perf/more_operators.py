"""The gated delta rule, for training and for serving, and the page tables of the caches beside it.

The state S [d, d] of a value head follows, token by token,

  S' = f_t S,   u_t = beta_t (v_t - S'^T k_t),   S = S' + k_t u_t^T,   o_t = scale S^T q_t,

with f_t = exp(log_f_t) the forget gate (1 without gates).  Value heads h * group .. h * group + group - 1 share query and key head h.
A server keeps a pool of states, a slot for each sequence, beside the pages of its attention caches; a sequence with no cached
tokens starts from a state of zeros.  Operators (``op`` of a case):

  fwd     o (and the last states) of whole sequences
  train   the same and all gradients, of a loss of o and the last states
  extend  chunks of new tokens for states in a pool, which are carried on in place
  step    one token, or a few drafted ones, for every sequence of a batch: the recurrent form
  plan    two steps of a server in which sequences end and others begin: page tables made to fit the requests' lengths, pages
          nobody needs put back on the stack of free ones, offsets of the packed new tokens, and the slot of each

``listed()`` names the cases, ``draw()`` gives further ones of the same ranges, ``prepare()`` makes what a program holds before the call,
``run()`` is one pass (``own``) or the same in elementary operations in 32 bits, ``exact()`` the definition token by token in 64 bits,
``work()`` the bytes and operations that a pass cannot do without.
"""
from __future__ import annotations

import math
import random

import torch

own = False

CHUNK = 64                                  # tokens that the plain form takes at a time
MAX_WORK = 4 * 16 * 8192 * 128              # tokens times value heads times d of a drawn case
EXACT_STATES = 3 << 30                      # 64-bit state elements that exact() holds at once


def _case(op, S, H, L, d=128, group=1, dtype="bf16", gates=True, layout="packed", states=False, shortest=None, spread="same"):
    return dict(op=op, S=S, H=H, group=group, L=L, shortest=L if shortest is None else shortest, spread=spread, d=d, dtype=dtype,
                gates=gates, layout=layout, states=states)


def _plan(S, per_seq, cached, new, page, spare):
    return dict(op="plan", S=S, per_seq=per_seq, cached=cached, new=new, page=page, spare=spare)


def listed():
    return [
        # a batch of long sequences, forward only (evaluation, or the forward of a recomputing step)
        dict(name="fwd_4x16x8192", **_case("fwd", 4, 16, 8192, layout="bhld")),
        # one long prompt read at once, few heads, its last state kept
        dict(name="fwd_1x8x16384_state", **_case("fwd", 1, 8, 16384, layout="blhd", states=True)),
        # a training step on the same batch; the largest
        dict(name="train_4x16x8192", **_case("train", 4, 16, 8192, layout="bhld")),
        # sequences of all lengths packed into one batch, value heads in pairs, states carried from segment to segment
        dict(name="train_packed_9x2999_group2", **_case("train", 9, 8, 2999, group=2, states=True, shortest=40, spread="ragged")),
        # a small fp32 step, as a check of a model's port runs it; no gates
        dict(name="train_2x3x300_d64_fp32", **_case("train", 2, 3, 300, d=64, dtype="fp32", gates=False, layout="blhd")),
        # a chunk of a long prompt
        dict(name="extend_chunk_1x16x512", **_case("extend", 1, 16, 512)),
        # a batch as a server runs it: one chunk of a prompt, everybody else one token; narrow heads, odd lengths
        dict(name="extend_mixed_12x701_d64", **_case("extend", 12, 16, 701, d=64, group=2, spread="one_long")),
        # one sequence decoding: latency
        dict(name="step_1x16", **_case("step", 1, 16, 1)),
        # a decoding batch: bound by memory
        dict(name="step_64x16_group2", **_case("step", 64, 16, 1, group=2)),
        # drafted tokens
        dict(name="step_drafts_16x16x5", **_case("step", 16, 16, 5, shortest=1, spread="ragged")),
        # a few sequences, short tables
        dict(name="plan_8x64", **_plan(8, 64, 3000, 12, 64, 100)),
        # many sequences with long tables, prompts among them, in a pool that is nearly used up
        dict(name="plan_500x2048", **_plan(500, 2048, 30000, 400, 16, 0)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: whole sequences or chunks of one token up to long ones (lengths on a logarithmic scale, odd ones among them),
    single and drafted tokens for batches of any size, tables from a few entries to a million."""
    op = rng.choice(["fwd", "train", "extend", "step", "plan"])
    if op == "plan":
        S, page = _log_int(rng, 1, 1000), rng.choice([16, 32, 64, 256])
        per_seq = _log_int(rng, 4, min(4096, 1000000 // S))
        cached = rng.randint(0, per_seq * page)
        return _plan(S, per_seq, cached, _log_int(rng, 1, max(1, min(2000, 200000 // S))), page, rng.choice([0, 3, 1000]))
    d = rng.choice([64, 128])
    dtype = "fp32" if rng.random() < 0.15 else "bf16"
    H, group = rng.choice([1, 2, 3, 4, 8, 16]), rng.choice([1, 1, 2, 4])
    gates = rng.random() < 0.8
    top = MAX_WORK // (H * group * d) // (16 if dtype == "fp32" else 1)       # tokens
    if op == "step":
        L = 1 if rng.random() < 0.6 else rng.randint(2, 8)
        return _case(op, _log_int(rng, 1, max(1, min(128, top // (16 * L)))), H, L, d=d, group=group, dtype=dtype, gates=gates,
                     shortest=rng.choice([1, L]), spread="ragged" if L > 1 else "same")
    L = _log_int(rng, 1 if op != "extend" else 9, min(16384 if op != "extend" else 4096, top))
    S = _log_int(rng, 1, max(1, min(16, top // L)))
    spread = "same" if S == 1 else rng.choice(["same", "ragged", "one_long"] if op == "extend" else ["same", "ragged"])
    layout = "packed" if op == "extend" or spread != "same" else rng.choice(["packed", "bhld", "blhd"])
    return _case(op, S, H, L, d=d, group=group, dtype=dtype, gates=gates, layout=layout, states=op != "extend" and rng.random() < 0.5,
                 shortest=rng.choice([1, max(1, L // 10)]) if spread == "ragged" else L, spread=spread)


def _lengths(case):
    """Tokens of each sequence: all alike, anything between the shortest and the longest (which occurs), or one chunk among single tokens."""
    S, rng = case["S"], random.Random(f"{case['S']} {case['shortest']} {case['L']}")
    n = [case["L"]] * S
    if case["spread"] == "ragged":
        n = [rng.randint(case["shortest"], case["L"]) for _ in range(S)]
    elif case["spread"] == "one_long":
        n = [1] * S
    n[S // 3] = case["L"]
    return n


def prepare(case, seed):
    return _prepare_plan(case, seed) if case["op"] == "plan" else _prepare_delta(case, seed)


def _prepare_delta(case, seed):
    op, S, H, G, d = case["op"], case["S"], case["H"], case["group"], case["d"]
    dev = torch.device("cuda")
    td = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *shape: torch.randn(*shape, device=dev, generator=gen)
    n = _lengths(case)
    T, V = sum(n), H * G
    if case["layout"] == "packed":
        dims = lambda heads, *more: (T, heads, *more)
    elif case["layout"] == "blhd":
        dims = lambda heads, *more: (S, case["L"], heads, *more)
    else:
        dims = lambda heads, *more: (S, heads, case["L"], *more)
    unit = lambda x: torch.nn.functional.normalize(x, dim=-1)
    s = dict(case=case, scale=d ** -0.5, T=T, max_len=max(n), cu=None, log_f=None, state=None, ws=None,
             q=unit(rn(*dims(H, d))).to(td), k=unit(rn(*dims(H, d))).to(td), v=rn(*dims(V, d)).to(td),
             beta=torch.sigmoid(rn(*dims(V))).to(td))
    if case["gates"]:      # of a few per cent a token
        s["log_f"] = torch.nn.functional.logsigmoid(rn(*dims(V)) + 3.0).to(td)
    if case["layout"] == "packed":
        s["cu"] = torch.tensor([0] + [sum(n[:i + 1]) for i in range(S)], dtype=torch.int32, device=dev)
    if op in ("extend", "step"):
        slots = S + 3                                              # a few belong to nobody
        s["states"] = 0.2 * rn(slots, V, d, d)
        s["slots"] = torch.randperm(slots, device=dev, generator=gen)[:S].to(torch.int32).contiguous()
        s["cached"] = torch.randint(0, 3, (S,), device=dev, generator=gen).to(torch.int32) * (1 if op == "extend" else 0) + (0 if op == "extend" else 7)
    elif case["states"]:
        s["state"] = 0.2 * rn(S, V, d, d)
    if op == "train":      # gradients as a mean over many tokens gives them
        s["d_o"] = (1e-3 * rn(*dims(V, d))).to(td)
        s["d_state"] = 1e-3 * rn(S, V, d, d) if case["states"] else None
    if own:      # the scratch memory that a program keeps
        import paper_2505_16381_amd as pa
        dt = pa.PATH_BF16 if case["dtype"] == "bf16" else pa.PATH_F32
        s["ws"] = torch.empty(pa.path_delta_workspace_bytes(S, T, max(n), H, G, d, dt, training=op == "train"), dtype=torch.uint8, device=dev)
    return s


def _prepare_plan(case, seed):
    """Lengths of two steps between which some sequences end, others begin, and the rest go on; in the pool, pages for the longer of the two
    steps and `spare` more, most of the first step's already in the table."""
    S, P, page = case["S"], case["per_seq"], case["page"]
    dev = torch.device("cuda")
    rng = random.Random(f"{S} {P} {case['cached']}")
    room = P * page
    steps = []
    long = [rng.randint(case["cached"] // 2, case["cached"]) for _ in range(S)]
    new = [rng.choice([1, 1, rng.randint(1, case["new"])]) for _ in range(S)]
    kind = [rng.choice(["on", "on", "end", "begin"]) for _ in range(S)]
    steps.append(([0 if x == "begin" else a for x, a in zip(kind, long)], [0 if x == "begin" else b for x, b in zip(kind, new)]))
    steps.append(([0 if x != "on" else min(a + b, room) for x, a, b in zip(kind, long, new)], [0 if x == "end" else 1 if x == "on" else rng.randint(1, case["new"]) for x in kind]))
    pages = [[min(P, -(-(a + b) // page)) for a, b in zip(*step)] for step in steps]
    pool = max(1, max(sum(p) for p in pages) + case["spare"] - (S // 50 if case["spare"] == 0 else 0))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    order = torch.randperm(pool, device=dev, generator=gen).to(torch.int32)
    held = torch.tensor([min(P, -(-a // page)) for a in steps[0][0]], device=dev)      # pages of the cached tokens lie anywhere
    at = torch.arange(P, device=dev)
    before = torch.cumsum(held, 0) - held
    index = before[:, None] + at
    table = torch.where((at < held[:, None]) & (index < pool), order[index.clamp(max=pool - 1)], -1).to(torch.int32).contiguous()
    used = min(pool, sum(min(P, -(-a // page)) for a in steps[0][0]))
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    free = torch.zeros(pool, dtype=torch.int32, device=dev)
    free[:pool - used] = order[used:]
    s = dict(case=case, table=table, free=free, count=ints([pool - used]), steps=[(ints(a), ints(b), sum(b)) for a, b in steps], ws=None)
    if own:
        import paper_2505_16381_amd as pa
        s["ws"] = torch.empty(max(256, pa.path_paged_plan_workspace_bytes(S, P, max(sum(b) for _, b in steps))), dtype=torch.uint8, device=dev)
    return s


def run(s):
    op = s["case"]["op"]
    if not own:
        return _plain_steps(s) if op == "plan" else _plain_serve(s) if op in ("extend", "step") else _plain_whole(s)
    import paper_2505_16381_amd as pa
    if op == "plan":
        out = ()
        for cached, new, T in s["steps"]:
            out += pa.path_paged_plan(cached, new, s["table"], s["free"], s["count"], T, s["case"]["page"], workspace=s["ws"])
        return (*out, s["table"], s["free"], s["count"])
    x = (s["q"], s["k"], s["v"], s["beta"])
    if op in ("extend", "step"):
        o = pa.path_delta_extend(*x, s["states"], s["slots"], s["cached"], s["cu"], s["max_len"], log_f=s["log_f"], scale=s["scale"], workspace=s["ws"])
        return o, s["states"]
    how = dict(log_f=s["log_f"], scale=s["scale"], state_in=s["state"], workspace=s["ws"])
    if s["cu"] is not None:
        how.update(cu_seqlens=s["cu"], max_len=s["max_len"])
    else:
        how.update(layout=pa.PATH_LAYOUT_BLHD if s["case"]["layout"] == "blhd" else pa.PATH_LAYOUT_BHLD)
    if op == "fwd":
        return pa.path_delta_fwd(*x, final_state=s["case"]["states"], **how)
    out = pa.path_delta_train_fwd(*x, final_state=s["case"]["states"], **how)
    out = out if s["case"]["states"] else (out,)
    return (*out, *pa.path_delta_train_bwd(*x, s["d_o"], d_state_out=s["d_state"], **how))


# ---- the plain forms ------------------------------------------------------------------------------------------------

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


def _chunks(q, k, v, beta, log_f, S, scale):
    """o [N,V,L,d] and the last states, of q, k, v [N,V,L,d], beta, log_f [N,V,L] and the first states S [N,V,d,d], 64 tokens at a time:
    within a chunk (I + beta tril(D K K^T)) U = beta (V - gamma K S), D_ri = exp(b_r - b_i), b the running sums of log_f."""
    L, d = q.shape[-2:]
    C = min(CHUNK, 1 << max(0, L - 1).bit_length())
    short = -L % C
    pad = lambda x: torch.nn.functional.pad(x, (0, 0, 0, short)).unflatten(2, (-1, C))
    q, k, v = pad(q), pad(k), pad(v)                                                     # [N, V, chunks, C, d]
    beta, b = pad(beta[..., None])[..., 0], torch.cumsum(pad(log_f[..., None])[..., 0], -1)
    lower = torch.ones(C, C, device=q.device, dtype=torch.bool).tril()
    D = torch.exp((b[..., :, None] - b[..., None, :]).masked_fill(~lower, -math.inf))
    inverse = _block_inverses((beta[..., None] * D * (k @ k.mT)).tril(-1), C)[..., 0, :, :] * beta[..., None, :]
    gamma, rest = torch.exp(b)[..., None], torch.exp(b[..., -1:] - b)[..., None]
    W, Ut = inverse @ (gamma * k), inverse @ v
    M, qg, kg, last = scale * D * (q @ k.mT), scale * gamma * q, (rest * k).mT, gamma[..., -1:, :]
    out = []
    for c in range(q.shape[2]):
        U = Ut[:, :, c] - W[:, :, c] @ S
        out.append(qg[:, :, c] @ S + M[:, :, c] @ U)
        S = last[:, :, c] * S + kg[:, :, c] @ U
    return torch.stack(out, 2).flatten(2, 3)[:, :, :L], S


def _rows(s):
    """Sequences and places of the tokens of a packed batch, padded to the longest, and which of them are there."""
    cu = s["cu"].long()
    a = torch.arange(s["max_len"], device=cu.device)
    there = a < (cu[1:] - cu[:-1])[:, None]
    return (cu[:-1, None] + a).clamp(max=s["T"] - 1), there


def _wide(s, x, shared):
    """A tensor of the case's layout as [N, V, L, ..] in 32 bits, padded with zeros, shared heads repeated."""
    layout, G = s["case"]["layout"], s["case"]["group"]
    x = x.float()
    if layout == "packed":
        at, there = _rows(s)
        x = (x[at] * there.view(*there.shape, *[1] * (x.dim() - 1))).transpose(1, 2)
    elif layout == "blhd":
        x = x.transpose(1, 2)
    return x.repeat_interleave(G, 1) if shared else x


def _narrow(s, x):
    """[N, V, L, ..] in the case's layout."""
    layout = s["case"]["layout"]
    if layout == "packed":
        return x.transpose(1, 2)[_rows(s)[1]]
    return x.transpose(1, 2).contiguous() if layout == "blhd" else x


def _plain_whole(s):
    case = s["case"]
    td = s["q"].dtype
    given = [s[x] for x in ("q", "k", "v", "beta")] + [x for x in (s["log_f"], s["state"]) if x is not None]
    train = case["op"] == "train"
    if train:
        given = [x.float().requires_grad_() for x in given]
    q, k, v, beta, *more = given
    with torch.set_grad_enabled(train):
        v, beta = _wide(s, v, False), _wide(s, beta, False)
        log_f = _wide(s, more[0], False) if s["log_f"] is not None else torch.zeros_like(beta)
        S = more[-1] if s["state"] is not None else torch.zeros(*v.shape[:2], case["d"], case["d"], device=v.device)
        o, S = _chunks(_wide(s, q, True), _wide(s, k, True), v, beta, log_f, S, s["scale"])
        o = _narrow(s, o)
        if train:
            loss = (o * s["d_o"].float()).sum() + ((S * s["d_state"]).sum() if s["d_state"] is not None else 0.0)
            grads = torch.autograd.grad(loss, given)
    out = (o.detach().to(td), S.detach()) if case["states"] else (o.detach().to(td),)
    if train:
        return (*out, *[g.to(x) for g, x in zip(grads, [td] * (5 if s["log_f"] is not None else 4) + [torch.float32])])
    return out if case["states"] else out[0]


def _plain_serve(s):
    slots = s["slots"].long()
    S = s["states"][slots] * (s["cached"] > 0)[:, None, None, None]
    v, beta = _wide(s, s["v"], False), _wide(s, s["beta"], False)
    log_f = _wide(s, s["log_f"], False) if s["log_f"] is not None else torch.zeros_like(beta)
    o, S = _chunks(_wide(s, s["q"], True), _wide(s, s["k"], True), v, beta, log_f, S, s["scale"])
    s["states"][slots] = S
    return _narrow(s, o).to(s["q"].dtype), s["states"]


def _plain_plan(cached, new, table, free, count, T, page):
    """The table's entries behind the tokens of cached + new go back to the stack of free pages, entries that the new tokens want are taken
    off its top, both in the order of the table; a page that is not there to take leaves a hole (-1)."""
    P, pool = table.shape[1], free.shape[0]
    dev = table.device
    n = cached.long().clamp(min=0)
    cu = torch.nn.functional.pad(torch.cumsum(new.long().clamp(min=0), 0), (1, 0)).clamp(max=T)
    have, want = (n + page - 1) // page, ((n + cu[1:] - cu[:-1] + page - 1) // page).clamp(max=P)
    j = torch.arange(P, device=dev)
    valid = (table >= 0) & (table < pool)
    behind = j >= want[:, None]
    back, need = (valid & behind).flatten(), (~valid & (j >= have[:, None]) & ~behind).flatten()
    base = count.long().clamp(0, pool)
    place = torch.where(back, base + torch.cumsum(back, 0) - 1, pool).clamp(max=pool)       # past the stack's end: nowhere
    stack = torch.cat([free, free[:1]]).scatter(0, place, torch.where(place < pool, table.flatten(), free[0]))[:pool]
    top = (base + back.sum()).clamp(max=pool)
    place = top - torch.cumsum(need, 0)
    got = need & (place >= 0)
    filled = torch.where(got, stack[place.clamp(0, pool - 1)], -1).to(torch.int32)
    table.copy_(torch.where(behind, -1, torch.where(need.view_as(table), filled.view_as(table), table)))
    free.copy_(stack)
    count.copy_((top - need.sum()).clamp(min=0))
    t = torch.arange(T, device=dev)
    seq = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    there = seq < len(n)
    seq = seq.clamp(max=len(n) - 1)
    pos = n[seq] + t - cu[seq]
    entry = table[seq, (pos // page).clamp(max=P - 1)].long()
    slot = torch.where(there & (pos < P * page) & (entry >= 0) & (entry < pool), entry * page + pos % page, -1)
    return cu.to(torch.int32), slot, (need & ~got).view_as(table).sum(1).to(torch.int32)


def _plain_steps(s):
    plan = lambda step: _plain_plan(step[0], step[1], s["table"], s["free"], s["count"], step[2], s["case"]["page"])
    return (*plan(s["steps"][0]), *plan(s["steps"][1]), s["table"], s["free"], s["count"])


# ---- the definition, token by token, in 64 bits ---------------------------------------------------------------------

def exact(case, seed):
    """The recurrence, and for gradients its reverse, a few heads at a time so that the state behind every token can be kept."""
    if case["op"] == "plan":
        return None
    s = prepare(case, seed)
    V, G, d, L, layout = case["H"] * case["group"], case["group"], case["d"], s["max_len"], case["layout"]
    n = _lengths(case)
    train, serve = case["op"] == "train", case["op"] in ("extend", "step")
    rows = [(i, h) for i in range(case["S"]) for h in range(V)]
    at_once = max(1, EXACT_STATES // (L * d * d)) if train else len(rows)
    if -(-len(rows) // at_once) * L > 60000:
        return None
    dev, f64 = s["q"].device, torch.float64
    first = [sum(n[:i]) for i in range(case["S"])]

    def view(x, i):      # [tokens, heads, ..] of sequence i
        return x[first[i]:first[i] + n[i]] if layout == "packed" else x[i] if layout == "blhd" else x[i].transpose(0, 1)

    new = lambda like: torch.zeros(like.shape, dtype=f64, device=dev)
    names = ["q", "k", "v", "beta"] + (["log_f"] if case["gates"] else [])
    o, grad = new(s["v"]), {x: new(s[x]) for x in names} if train else {}
    if serve:
        last = s["states"].double()
        begin = last[s["slots"].long()] * (s["cached"] > 0)[:, None, None, None]
    else:
        begin = s["state"].double() if s["state"] is not None else torch.zeros(case["S"], V, d, d, dtype=f64, device=dev)
        last = torch.zeros_like(begin)
    d_begin = torch.zeros_like(begin)
    for r0 in range(0, len(rows), at_once):
        mine = rows[r0:r0 + at_once]
        N = len(mine)

        def take(x, shared):      # [L, N, ..], zeros behind a sequence's end
            y = torch.zeros(L, N, *x.shape[2 if layout == "packed" else 3:], dtype=f64, device=dev)
            for j, (i, h) in enumerate(mine):
                y[:n[i], j] = view(x, i)[:, h // G if shared else h].double()
            return y

        q, k, v, beta = take(s["q"], True), take(s["k"], True), take(s["v"], False), take(s["beta"], False)
        f = torch.exp(take(s["log_f"], False)) if case["gates"] else torch.ones_like(beta)
        S = torch.stack([begin[i, h] for i, h in mine])
        kept = torch.empty(L + 1 if train else 1, N, d, d, dtype=f64, device=dev)
        kept[0] = S
        y = torch.empty(L, N, d, dtype=f64, device=dev)
        for t in range(L):
            S = S * f[t, :, None, None]
            u = beta[t, :, None] * (v[t] - (S * k[t, :, :, None]).sum(1))
            S = S + k[t, :, :, None] * u[:, None]
            y[t] = s["scale"] * (S * q[t, :, :, None]).sum(1)
            if train:
                kept[t + 1] = S
        for j, (i, h) in enumerate(mine):
            view(o, i)[:, h] = y[:n[i], j]
            last[int(s["slots"][i]) if serve else i, h] = S[j]
        if not train:
            continue
        dO = take(s["d_o"], False)
        Gs = torch.stack([s["d_state"][i, h].double() for i, h in mine]) if s["d_state"] is not None else torch.zeros(N, d, d, dtype=f64, device=dev)
        dq, dk, dv, db, dl = (torch.zeros_like(x) for x in (q, k, v, beta, beta))
        for t in range(L - 1, -1, -1):
            S, old = kept[t + 1], kept[t] * f[t, :, None, None]
            dq[t] = s["scale"] * (S * dO[t, :, None]).sum(-1)
            Gs = Gs + s["scale"] * q[t, :, :, None] * dO[t, :, None]
            e = v[t] - (old * k[t, :, :, None]).sum(1)
            du = (Gs * k[t, :, :, None]).sum(1)
            db[t] = (du * e).sum(-1)
            dv[t] = beta[t, :, None] * du
            dk[t] = (Gs * (beta[t, :, None] * e)[:, None]).sum(-1) - (old * dv[t, :, None]).sum(-1)
            Gs = Gs - k[t, :, :, None] * dv[t, :, None]
            dl[t] = (Gs * old).sum((-1, -2))
            Gs = Gs * f[t, :, None, None]
        for j, (i, h) in enumerate(mine):
            for x, g in zip(("q", "k", "v", "beta", "log_f"), (dq, dk, dv, db, dl)):
                if x in grad:
                    view(grad[x], i)[:, h // G if x in "qk" else h] += g[:n[i], j]
            d_begin[i, h] = Gs[j]
        del kept
    if serve:
        return o, last
    out = (o, last) if case["states"] else (o,)
    if train:
        return (*out, *[grad[x] for x in names], *([d_begin] if case["states"] else []))
    return out if case["states"] else o


def work(case):
    """Each input read once and each output written once.  Per token and value head, 4 d^2 operations for reading the state and writing to
    it, 2 d^2 for its prediction of the value; the gradients twice that."""
    if case["op"] == "plan":      # tables, lengths and offsets; a slot of each new token (about a third of the longest for each sequence)
        return {"bytes": 2.0 * (8 * case["S"] * case["per_seq"] + 16 * case["S"] + 8 * max(1, case["S"] * case["new"] // 3)), "flops": 1.0}
    op, H, G, d, S = case["op"], case["H"], case["group"], case["d"], case["S"]
    es, g, T = (2 if case["dtype"] == "bf16" else 4), (1 if case["gates"] else 0), sum(_lengths(case))
    inputs = T * (2 * H * d + H * G * (d + 1 + g)) * es
    state = 4 * S * H * G * d * d
    nbytes = inputs + T * H * G * d * es + state * (2 if op in ("extend", "step") or case["states"] else 0)
    flops = 6.0 * d * d * T * H * G
    if op == "train":      # the inputs and the gradient of o read, all gradients written
        nbytes += 2 * inputs + T * H * G * d * es + (2 * state if case["states"] else 0)
        flops *= 3
    return {"bytes": float(nbytes), "flops": flops}
