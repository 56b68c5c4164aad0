"""Served calls of the gated delta rule (path_delta_extend), alone and as a server runs them: page tables, attention over paged caches and states in a pool, step by step.
Bars as in test_gpu_delta.py."""
import math
import random

import pytest

import delta_model as dm
from test_gpu_delta import close, to_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    import paper_2505_16381_amd as pa
    assert torch.cuda.is_available()
    pa.load_library()
    return torch, pa


def pool(torch, nseq, V, d, seed=0, extra=3):
    g = torch.Generator().manual_seed(seed)
    states = 0.3 * torch.randn(nseq + extra, V, d, d, generator=g)
    return states, torch.randperm(nseq + extra, generator=g)[:nseq].to(torch.int32)


def serve(gpu, lengths, cached, H=2, G=1, d=64, dtype="bf16", gates=True, seed=0, slots=None, tail=0, max_new=None, change=None):
    torch, pa = gpu
    x = dm.batch(lengths, H, G, d, dtype, gates, seed, tail=tail)
    if change:
        change(torch, x)
    states, own = pool(torch, len(lengths), H * G, d, seed)
    slots = own if slots is None else torch.tensor(slots, dtype=torch.int32)
    y, scale, cu = to_gpu(x), d ** -0.5, x["cu"].tolist()
    st = states.cuda()
    max_new = max_new or max(1, max(lengths))
    ws = torch.full((pa.path_delta_workspace_bytes(len(lengths), x["q"].shape[0], max_new, H, G, d, 1 if dtype == "bf16" else 0),), 255, dtype=torch.uint8, device="cuda")
    o = torch.full_like(y["v"], 5.0)
    pa.path_delta_extend(y["q"], y["k"], y["v"], y["beta"], st, slots.cuda(), torch.tensor(cached, dtype=torch.int32, device="cuda"), y["cu"], max_new, log_f=y["log_f"], scale=scale, o=o,
                         workspace=ws)
    there = [0 <= s < len(states) for s in slots.tolist()]
    first = torch.stack([states[s] if ok and c > 0 else torch.zeros_like(states[0]) for s, ok, c in zip(slots.tolist(), there, cached)])
    want_o, want_last = dm.forward(x, scale, first)
    assert (o[cu[-1]:] == 5.0).all()
    close(torch, "o", o, want_o, cu, dtype == "fp32")
    want = states.double().clone()
    for s, (slot, ok, n) in enumerate(zip(slots.tolist(), there, lengths)):
        if ok and n > 0:
            want[slot] = want_last[s]
    touched = [slot for slot, ok, n in zip(slots.tolist(), there, lengths) if ok and n > 0]
    rest = [i for i in range(len(states)) if i not in touched]
    assert torch.equal(st.cpu()[rest], states[rest])
    if touched:
        close(torch, "state", st[touched], want[touched], cu, dtype == "fp32")
    return o


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lengths", [[1], [1] * 9, [3, 0, 8, 1], [8], [9], [64], [65], [1, 200, 1, 0, 8, 9], [100, 129]], ids=str)
def test_extend(gpu, d, dtype, lengths):
    rng = random.Random(d + len(lengths))
    serve(gpu, lengths, [rng.choice([0, 1, 500]) for _ in lengths], 2, 1, d, dtype, seed=len(lengths))


@pytest.mark.parametrize("H,G", [(1, 1), (3, 2), (2, 5)])
@pytest.mark.parametrize("gates", [True, False])
@pytest.mark.parametrize("d", [64, 128])
def test_heads_and_gates(gpu, H, G, gates, d):
    serve(gpu, [1, 5, 90, 2], [4, 0, 9, 1], H, G, d, "bf16", gates, seed=H)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_long_prompts(gpu, dtype):
    """Prompts of few heads, cut into segments; beside short ones, in fresh, carried and no slots."""
    serve(gpu, [2500, 1, 800, 0], [7, 7, 0, 7], 1, 2, 64, dtype, seed=1)
    serve(gpu, [2500, 9, 2400], [0, 7, 7], 1, 1, 128, dtype, seed=2, slots=[3, -1, 0])
    serve(gpu, [2400], [7], 1, 1, 64, dtype, seed=3, max_new=10000)


def test_slots_that_are_none(gpu):
    """A sequence whose slot is outside the pool starts from zeros and is not kept."""
    serve(gpu, [1, 4, 70, 2, 80], [3, 3, 3, 3, 3], 2, 2, 64, slots=[-1, 2, 99, 0, 1], seed=3)
    serve(gpu, [70, 80], [3, 3], 2, 1, 128, slots=[-5, 1 << 30], seed=3)


def test_rows_and_bounds(gpu):
    """Rows behind the last sequence are left; a bound well above the lengths, which chooses other kernels, changes nothing but rounding."""
    serve(gpu, [1, 2, 1], [1, 0, 7], 2, 2, 64, tail=9, seed=5)
    serve(gpu, [1, 2, 1], [1, 0, 7], 2, 2, 64, tail=90, max_new=90, seed=5)
    serve(gpu, [5], [2], 2, 2, 64, tail=90, max_new=90, seed=5)


def forgets(torch, x):
    x["log_f"][2] = -math.inf
    x["beta"][1] = 0.0
    x["beta"][3] = 2.0


def test_values(gpu):
    for lengths in ([8, 8], [80, 30]):
        serve(gpu, lengths, [5, 5], 2, 1, 64, change=forgets, seed=7)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_token_by_token_is_the_chunk(gpu, dtype):
    """Forty tokens one at a time, in drafts, and at once leave the same states."""
    torch, pa = gpu
    x = dm.batch([40, 40], 2, 2, 64, dtype, seed=2)
    y = to_gpu(x)
    states, slots = pool(torch, 2, 4, 64)
    want_o, want_last = dm.forward(x, 0.125, states[slots.long()])
    for step in (1, 5, 8, 13, 40):
        st, outs = states.cuda(), []
        for a in range(0, 40, step):
            m = min(step, 40 - a)
            pick = torch.tensor([*range(a, a + m), *range(40 + a, 40 + a + m)], device="cuda")
            part = {n: y[n][pick].contiguous() for n in ("q", "k", "v", "beta", "log_f")}
            cu = torch.tensor([0, m, 2 * m], dtype=torch.int32, device="cuda")
            o = pa.path_delta_extend(part["q"], part["k"], part["v"], part["beta"], st, slots.cuda(), torch.full((2,), a + 1, dtype=torch.int32, device="cuda"), cu, m, log_f=part["log_f"],
                                     scale=0.125)
            outs.append((pick, o))
        o = torch.empty_like(y["v"])
        for pick, part in outs:
            o[pick] = part
        close(torch, "o", o, want_o, [0, 40, 80], dtype == "fp32")
        close(torch, "state", st[slots.long()], want_last, [0, 40, 80], dtype == "fp32")


def test_no_token_before_one_that_is_not_finite(gpu):
    """Token by token, what is not finite shows in no row before it, and in no other head or sequence."""
    torch, pa = gpu
    for n in ("q", "k", "v", "beta", "log_f"):
        x = dm.batch([8, 8], 3, 1, 64, seed=2)
        y = to_gpu(x)
        call = lambda st: pa.path_delta_extend(y["q"], y["k"], y["v"], y["beta"], st, torch.tensor([1, 0], dtype=torch.int32, device="cuda"),
                                               torch.tensor([1, 1], dtype=torch.int32, device="cuda"), y["cu"], 8, log_f=y["log_f"])
        states = pool(torch, 2, 3, 64)[0].cuda()
        a, b = states.clone(), states.clone()
        o = call(a)
        y[n][4, 1] = math.nan
        o1 = call(b)
        keep = torch.ones(16, 3, dtype=torch.bool, device="cuda")
        keep[4:8, 1] = False
        assert torch.equal(o1[keep], o[keep]), n
        assert torch.equal(b[0], a[0]) and torch.equal(b[1, [0, 2]], a[1, [0, 2]])


def test_captured(gpu):
    """Single tokens, captured, follow slots, lengths and states through the replays."""
    torch, pa = gpu
    for lengths in ([1, 1, 1], [1, 60, 8]):
        x = dm.batch(lengths, 2, 2, 64, seed=1)
        y, T = to_gpu(x), sum(lengths)
        states, slots = pool(torch, 3, 4, 64)
        st, sl, cached = states.cuda(), slots.cuda(), torch.tensor([0, 3, 9], dtype=torch.int32, device="cuda")
        ws = torch.empty(pa.path_delta_workspace_bytes(3, T, max(lengths), 2, 2, 64, 1), dtype=torch.uint8, device="cuda")
        call = lambda st, ws: pa.path_delta_extend(y["q"], y["k"], y["v"], y["beta"], st, sl, cached, y["cu"], max(lengths), log_f=y["log_f"], workspace=ws)
        call(st.clone(), ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o = call(st, ws)
        ref = st.clone()
        for i in range(4):
            z = to_gpu(dm.batch(lengths, 2, 2, 64, seed=20 + i))
            for n in ("q", "k", "v", "beta", "log_f"):
                y[n].copy_(z[n])
            sl.copy_(torch.randperm(6, device="cuda")[:3].to(torch.int32))
            cached.copy_(torch.randint(0, 2, (3,), device="cuda").to(torch.int32))
            want = call(ref, torch.full_like(ws, 255))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, want) and torch.equal(st, ref)


@pytest.mark.parametrize("gates", [True, False])
def test_a_server(gpu, gates):
    """Tables, attention layer and recurrent layer together, over a server's steps with prompts, single tokens and drafts of which some are dropped, against both layers on the
    whole sequences at once.  The recurrent layer takes tokens only once they stay: drafts go through the attention alone."""
    torch, pa = gpu
    H, d, page, nseq, P = 2, 64, 16, 4, 20
    rng = random.Random(5)
    lengths = [90, 33, 150, 64]
    g = torch.Generator(device="cuda").manual_seed(3)
    unit = lambda *s: torch.nn.functional.normalize(torch.randn(*s, device="cuda", generator=g), dim=-1)
    data = []
    for n in lengths:
        data.append(dict(q=torch.randn(n, H, d, device="cuda", generator=g).bfloat16(), k=torch.randn(n, H, d, device="cuda", generator=g).bfloat16(),
                         v=torch.randn(n, H, d, device="cuda", generator=g).bfloat16(), w=unit(n, H, d).bfloat16(), dq=unit(n, H, d).bfloat16(),
                         beta=torch.sigmoid(torch.randn(n, H, device="cuda", generator=g)).bfloat16(),
                         log_f=torch.nn.functional.logsigmoid(torch.randn(n, H, device="cuda", generator=g) + 3).bfloat16()))
    pages = 60
    kpages, vpages = torch.full((pages, H, page, d), math.nan, device="cuda", dtype=torch.bfloat16), torch.full((pages, H, page, d), math.nan, device="cuda", dtype=torch.bfloat16)
    cpages = torch.full((pages, H, page), math.nan, device="cuda") if gates else None
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    table, free, count = torch.full((nseq, P), -1, dtype=torch.int32, device="cuda"), torch.randperm(pages, device="cuda").to(torch.int32), i32([pages])
    states, slots = torch.full((nseq + 2, H, d, d), math.nan, device="cuda"), i32([3, 0, 5, 1])
    done = [0] * nseq
    attn, rec = [[] for _ in range(nseq)], [[] for _ in range(nseq)]
    while any(a < b for a, b in zip(done, lengths)):
        left = [b - a for a, b in zip(done, lengths)]
        new = [min(n, rng.choice([0, 1, 1, 3, 40])) for n in left]
        T = sum(new)
        if T == 0:
            continue
        cached, fresh = i32(done), i32(new)
        cu, slot_map, missing = pa.path_paged_plan(cached, fresh, table, free, count, T, page)
        cat = lambda n: torch.cat([x[n][a:a + m] for x, a, m in zip(data, done, new)]).contiguous()
        kvwb = (cat("k"), cat("v"), cat("w"), cat("beta"))
        lf = cat("log_f") if gates else None
        how = (kpages, vpages, table, cached, cu, max(new), max(1, max(done)))
        drafts = rng.random() < 0.4 and max(new) <= 3
        if drafts:      # looked at, and dropped: nothing is appended, the pages go back with the next plan
            pa.path_paged_attn(cat("q"), *kvwb, *how, log_f=lf, cpages=cpages)
            continue
        o, _ = pa.path_paged_extend(cat("q"), *kvwb, *how, log_f=lf, cpages=cpages)
        r = pa.path_delta_extend(cat("dq"), cat("w"), cat("v"), cat("beta"), states, slots, cached, cu, max(new), log_f=lf)
        assert missing.sum() == 0 and (slot_map >= 0).all()
        assert torch.equal(vpages.transpose(1, 2).reshape(-1, H, d)[slot_map], kvwb[1])      # a new token's value lies in its slot
        at = 0
        for s, m in enumerate(new):
            attn[s].append(o[at:at + m])
            rec[s].append(r[at:at + m])
            at += m
        done = [a + b for a, b in zip(done, new)]
    _, _, _ = pa.path_paged_plan(i32([0] * nseq), i32([0] * nseq), table, free, count, 1, page)      # all sequences end
    assert count.item() == pages and sorted(free.tolist()) == list(range(pages)) and (table == -1).all()
    for s, x in enumerate(data):
        lf = x["log_f"] if gates else None
        whole = lambda n: x[n].transpose(0, 1)[None].contiguous()
        if gates:
            want, _ = pa.path_attn_fox_fwd(whole("q"), whole("k"), whole("v"), whole("w"), whole("beta"), whole("log_f"))
        else:
            want, _ = pa.path_attn_fwd(whole("q"), whole("k"), whole("v"), whole("w"), whole("beta"))
        got = torch.cat(attn[s]).float()
        assert (got - want[0].transpose(0, 1).float()).abs().max() <= 2 ** -6 * x["v"].abs().max()      # two roundings on each side, of weights and of results
        y = dict(q=x["dq"].cpu(), k=x["w"].cpu(), v=x["v"].cpu(), beta=x["beta"].cpu(), log_f=lf.cpu() if gates else None, cu=torch.tensor([0, lengths[s]]))
        close(torch, "o", torch.cat(rec[s]), dm.forward(y, d ** -0.5)[0], [0, lengths[s]], False)


@pytest.mark.parametrize("kind", ["stream", "handle"])
def test_made_tensors_are_of_the_given_stream(gpu, kind):
    torch, pa = gpu
    from test_gpu_paged_streams import stream_of
    y = to_gpu(dm.batch([30, 1], 2, 1, 64))
    states = torch.zeros(2, 2, 64, 64, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    sl, cached, table, free, count = i32([0, 1]), i32([0, 0]), i32([[-1] * 4] * 2), i32([0, 1, 2, 3]), i32([4])
    new = i32([30, 1])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    given = s if kind == "stream" else s.cuda_stream
    made = [pa.path_delta_extend(y["q"], y["k"], y["v"], y["beta"], states, sl, cached, y["cu"], 30, stream=given),
            *pa.path_paged_plan(cached, new, table, free, count, 31, 16, stream=given), pa.path_delta_fwd(y["q"], y["k"], y["v"], y["beta"], cu_seqlens=y["cu"], max_len=30, stream=given)]
    torch.cuda.synchronize()
    assert all(stream_of(torch, t) == s.cuda_stream for t in made)


def test_refusals(gpu):
    torch, pa = gpu
    y = to_gpu(dm.batch([3, 2], 2, 2, 64))
    st, i32 = torch.zeros(2, 4, 64, 64, device="cuda"), lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    good = dict(q=y["q"], k=y["k"], v=y["v"], beta=y["beta"], states=st, slots=i32([0, 1]), cached=i32([0, 0]), cu_new=y["cu"], max_new=3)
    pa.path_delta_extend(**good)
    for bad in (dict(k=y["k"].float()), dict(v=y["v"][:, :3].contiguous()), dict(beta=y["beta"].float()), dict(states=st.double()), dict(states=st[:, :3].contiguous()), dict(slots=i32([0])),
                dict(slots=i32([0, 1]).long()), dict(cached=i32([0, 0, 0])), dict(q=y["q"].transpose(0, 1).contiguous().transpose(0, 1)), dict(states=st.cpu()), dict(max_new=1 << 33)):
        with pytest.raises(ValueError):
            pa.path_delta_extend(**{**good, **bad})
    with pytest.raises(pa.PathAttnError):
        pa.path_delta_extend(**{**good, "max_new": 0})
    with pytest.raises(pa.PathAttnError):
        pa.path_delta_extend(**good, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(TypeError):
        pa.path_delta_extend(**{**good, **{n: good[n].half() for n in ("q", "k", "v", "beta")}})
