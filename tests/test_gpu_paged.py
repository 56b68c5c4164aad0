"""Paged caches on the GPU against the definition in 64 bits (paged_model.py).

Bars (e = half a step of bf16 = 2^-8, h = half a step of fp16 = 2^-11; inputs are standard normal, scale d^-1/2, so norms of q and k are below
1.6 sqrt(d) and scale |q| |k| below 2.6 sqrt(d)):
  o     bf16: every weight is rounded once (e of a mean of |v| <= 4.5) and the result once: 2 e max|v|.
        fp32: sums of up to 4000 terms of size one, of logits good to 1e-5: 1e-4.
  lse   bf16: x is a sum of two bf16 numbers, its rest 2^-16 of it: 2^-16 * 2.6 sqrt(d) = 4.5e-4, and as much for fp32 sums: 1e-3; chunks carry x and the keys
        through up to four tiles so: 2e-3.  fp32: 1e-4 (as above).
  keys  bf16: the result is rounded once, e |k'|; a chunk's cached keys meet a matrix of fp16 elements, rows of norm <= 2: an element is off by a
        deviation of 2 h / sqrt(3) = 6e-4, five of them 3e-3, and as much for the carried operands: e |k'| + 8e-3.  fp32: 1e-4.
  values and untouched slots: the bits."""
import math

import pytest

import paged_model as pm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    import paper_2505_16381_amd as pa
    assert torch.cuda.is_available()
    pa.load_library()
    return torch, pa


def to_gpu(torch, x):
    return {n: t.cuda() if t is not None else None for n, t in x.items()}


def call(pa, op, y, max_new, max_cached, scale, **more):
    kvwb = (y["k"], y["v"], y["w"], y["beta"])
    cache = (y["kpages"], y["vpages"], y["page_table"], y["cached"], y["cu_new"], max_new, max_cached)
    if op == "append":
        return pa.path_paged_append(*kvwb, *cache, log_f=y["log_f"], cpages=y["cpages"], **more)
    f = pa.path_paged_attn if op == "attn" else pa.path_paged_extend
    return f(y["q"], *kvwb, *cache, log_f=y["log_f"], cpages=y["cpages"], scale=scale, **more)


def bars(x):
    f32 = x["k"].element_size() == 4
    long = int((x["cu_new"][1:] - x["cu_new"][:-1]).max()) > 16
    vmax = max(float(x["v"].abs().max()) if x["v"].numel() else 0.0, float(x["vpages"].nan_to_num().abs().max()))
    return dict(o=1e-4 if f32 else 2 ** -7 * vmax, lse=1e-4 if f32 else 2e-3 if long else 1e-3, key=1e-4 if f32 else 8e-3, rel=0 if f32 else 2 ** -8)


def compare(torch, x, y, got, want, op):
    b = bars(x)
    o, lse, kp, vp, cp = want
    if op != "append":
        there = ~lse.isnan()
        go, gl = got[0].double().cpu(), got[1].double().cpu()
        assert not go[there].isnan().any() and not gl[there].isnan().any()
        assert (go - o)[there].abs().max() <= b["o"], (go - o)[there].abs().max()
        assert (gl - lse)[there].abs().max() <= b["lse"], (gl - lse)[there].abs().max()
    gk, gv = y["kpages"].cpu(), y["vpages"].cpu()
    if op == "attn":
        assert torch.equal(gk.view(torch.uint8), x["kpages"].view(torch.uint8))
    else:
        assert torch.equal(gk.isnan(), kp.isnan())
        off = (gk.double() - kp).nan_to_num().abs() - b["rel"] * kp.nan_to_num().abs()
        assert off.max() <= b["key"], off.max()
    assert torch.equal(gv.isnan(), vp.isnan())
    assert torch.equal(gv.double().nan_to_num(), vp.nan_to_num())
    if cp is not None:
        gc = y["cpages"].double().cpu()
        assert torch.equal(gc.isnan(), cp.isnan())
        assert (gc - cp).nan_to_num().abs().max() <= 1e-6 * max(1.0, float(cp.nan_to_num().abs().max())) * 16


def check(gpu, op, old, new, H=2, G=1, d=64, page=16, dtype="bf16", gates=False, seed=0, beta=None, bounds=(0, 0)):
    torch, pa = gpu
    x = pm.batch(old, new, H, G, d, page, dtype, gates, seed, beta=beta)
    y = to_gpu(torch, x)
    scale = d ** -0.5
    more = {}
    if op != "append":
        more = dict(o=torch.full_like(y["q"], 7.0), lse=torch.full(y["q"].shape[:2], 7.0, device="cuda"))
    got = call(pa, op, y, max(max(new), 1) + bounds[0], max(old) + bounds[1], scale, **more)
    torch.cuda.synchronize()
    compare(torch, x, y, got, pm.expect(x, scale, op), op)


FEW = [
    # old, new, H, G, d, page, gates
    ([0], [1], 1, 1, 64, 16, False),
    ([1], [1], 1, 1, 128, 16, False),
    ([15, 16, 17], [1, 1, 1], 2, 1, 64, 16, True),
    ([300, 0, 129, 5], [1, 16, 0, 3], 2, 1, 128, 32, False),
    ([300, 7, 129, 64], [5, 16, 1, 0], 1, 4, 64, 64, True),
    ([40, 500], [8, 3], 2, 8, 128, 128, False),
    ([33], [4], 3, 3, 64, 16, True),
    ([100], [1], 1, 64, 128, 256, False),
    ([3000], [2], 1, 2, 128, 16, True),
    ([2049, 1], [1, 1], 3, 1, 64, 4096, False),
]
CHUNKS = [
    ([0], [17], 1, 1, 64, 16, False),
    ([0], [200], 2, 1, 128, 64, True),
    ([70], [64], 2, 1, 64, 16, False),
    ([129, 1], [65, 63], 1, 2, 128, 32, True),
    ([300, 50, 0, 700, 5], [1, 130, 20, 0, 16], 2, 1, 64, 16, True),
    ([1100, 33], [257, 1], 1, 3, 128, 128, False),
    ([10, 20], [3, 5], 2, 32, 64, 16, False),      # 96 and 160 rows of few tokens
]


@pytest.mark.parametrize("op", ["attn", "append", "extend"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", FEW, ids=lambda c: "-".join(map(str, c[:1] + c[1:2])).replace(" ", ""))
def test_few_new_tokens(gpu, case, dtype, op):
    old, new, H, G, d, page, gates = case
    check(gpu, op, old, new, H, G, d, page, dtype, gates, seed=len(old) + sum(old) + d)


@pytest.mark.parametrize("op", ["attn", "append", "extend"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", CHUNKS, ids=lambda c: "-".join(map(str, c[:1] + c[1:2])).replace(" ", ""))
def test_chunks(gpu, case, dtype, op):
    old, new, H, G, d, page, gates = case
    check(gpu, op, old, new, H, G, d, page, dtype, gates, seed=len(old) + sum(old) + d)


@pytest.mark.parametrize("op", ["attn", "append", "extend"])
@pytest.mark.parametrize("beta", [0.0, 1.0, 2.0])
@pytest.mark.parametrize("new", [[9, 2], [130, 40]])
def test_projections_and_reflections(gpu, op, beta, new):
    """beta = 0 (nothing is carried), 1 (what a key has along w is gone: no inverse), 2 (reflections)."""
    check(gpu, op, [200, 31], new, 2, 1, 64, 32, "fp32", beta=beta, seed=7)
    check(gpu, op, [200, 31], new, 2, 1, 64, 32, "bf16", beta=beta, seed=7)


@pytest.mark.parametrize("op", ["attn", "append", "extend"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("new", [[3, 1, 2], [70, 1, 33]])
def test_holes_take_no_part(gpu, op, dtype, new):
    """Table entries outside the pool: at a sequence's start, inside, at its end (where tokens should have gone)."""
    torch, pa = gpu
    for gates in (False, True):
        x = pm.batch([150, 64, 100], new, 2, 2, 64, 16, dtype, gates, seed=3)
        x = pm.drop_pages(x, [(0, 0), (0, 4), (1, 1), (2, 6), (2, 7), (0, x["page_table"].shape[1] - 1)], x["kpages"].shape[0])
        y = to_gpu(torch, x)
        scale = 0.125
        got = call(pa, op, y, max(new), 150, scale)
        torch.cuda.synchronize()
        compare(torch, x, y, got, pm.expect(x, scale, op), op)


@pytest.mark.parametrize("op", ["attn", "extend"])
@pytest.mark.parametrize("new", [[2, 0, 1], [100, 0, 90]])
def test_rows_of_no_sequence_are_left(gpu, op, new):
    """A packed batch with rows before the first, between and behind the last sequence's; sequences without new tokens."""
    torch, pa = gpu
    x = pm.batch([40, 17, 3], new, 2, 1, 64, 16, "bf16", seed=5)
    T = x["k"].shape[0]
    for n in ("q", "k", "v", "w", "beta"):      # five rows of garbage on either side
        pad = torch.full((5, *x[n].shape[1:]), math.nan, dtype=x[n].dtype)
        x[n] = torch.cat([pad, x[n], pad])
    x["cu_new"] = x["cu_new"] + 5
    y = to_gpu(torch, x)
    o, lse = torch.full_like(y["q"], 3.0), torch.full(y["q"].shape[:2], -3.0, device="cuda")
    got = call(pa, op, y, max(new), 40, 0.125, o=o, lse=lse)
    torch.cuda.synchronize()
    assert got[0] is o and got[1] is lse
    assert (o[:5] == 3).all() and (o[5 + T:] == 3).all() and (lse[:5] == -3).all() and (lse[5 + T:] == -3).all()
    x["v"] = x["v"].nan_to_num()      # (its maximum sets the bar)
    compare(torch, x, y, got, pm.expect(x, 0.125, op), op)


@pytest.mark.parametrize("op", ["attn", "append", "extend"])
@pytest.mark.parametrize("new", [[1, 4], [90, 17]])
def test_loose_bounds_change_nothing_but_time(gpu, op, new):
    """max_new and max_cached far above the lengths: the ways may differ, the results hold."""
    check(gpu, op, [300, 45], new, 2, 1, 128, 64, "bf16", True, seed=11, bounds=(0, 19))
    torch, pa = gpu
    x = pm.batch([300, 45], new, 2, 1, 128, 64, "bf16", True, seed=11)
    spare = torch.full((2, 40), -1, dtype=torch.int32)      # room in the table for the bound
    x["page_table"] = torch.cat([x["page_table"], spare], 1).contiguous()
    y = to_gpu(torch, x)
    got = call(pa, op, y, 200, 2000, 0.09)
    torch.cuda.synchronize()
    compare(torch, x, y, got, pm.expect(x, 0.09, op), op)


@pytest.mark.parametrize("new", [[1], [80]])
def test_lengths_beyond_the_bounds_are_held_to_them(gpu, new):
    """cached above max_cached, cu_new above T: nothing is read or written out of range; what lies inside is as if the lengths were the bounds."""
    torch, pa = gpu
    x = pm.batch([100], new, 2, 1, 64, 16, "bf16", seed=2)
    want = pm.expect(x, 0.125, "attn")
    y = to_gpu(torch, x)
    y["cached"] = torch.tensor([10 ** 9], dtype=torch.int32, device="cuda")
    y["cu_new"] = torch.tensor([-7, 10 ** 9], dtype=torch.int32, device="cuda")
    got = call(pa, "attn", y, new[0], 100, 0.125)
    torch.cuda.synchronize()
    compare(torch, x, y, got, want, "attn")


def test_values_behind_the_end_never_show(gpu):
    """Infinities and NaN in slots behind a sequence's last token (batch() puts NaN there), in pages of nobody, and infinite VALUES of a later new token in a chunk of
    few tokens."""
    torch, pa = gpu
    x = pm.batch([37], [4], 1, 1, 64, 16, "bf16", seed=9, unused=math.inf)
    x["v"][3] = math.inf
    y = to_gpu(torch, x)
    o, lse = call(pa, "attn", y, 4, 37, 0.125)
    torch.cuda.synchronize()
    assert torch.isfinite(o[:3]).all() and torch.isfinite(lse).all() and torch.isinf(o[3]).all()


@pytest.mark.parametrize("old,new", [([200, 70], [1, 1]), ([200, 70], [100, 1]), ([900, 3], [6, 2])])
def test_a_captured_call_follows_the_lengths(gpu, old, new):
    """extend captured once and replayed while the program appends, in between eager work: every replay against eager calls on another cache."""
    torch, pa = gpu
    x = pm.batch([n + 3 * max(new) for n in old], new, 2, 2, 64, 16, "bf16", True, seed=4)
    x["cached"] = torch.tensor(old, dtype=torch.int32)
    y, z = to_gpu(torch, x), to_gpu(torch, x)
    cap = max(old) + 3 * max(new)
    ws = torch.empty(pa.path_paged_workspace_bytes(len(old), sum(new), max(new), cap, 2, 2, 64, pa.PATH_BF16), dtype=torch.uint8, device="cuda")
    counts = torch.tensor(new, dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        o, lse = torch.empty_like(y["q"]), torch.empty(y["q"].shape[:2], device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call(pa, "extend", y, max(new), cap, 0.1, o=o, lse=lse, workspace=ws)
    for step in range(3):
        for n in ("q", "k", "v", "w", "beta", "log_f"):
            fresh = torch.roll(x[n], step, 0).cuda()
            y[n].copy_(fresh)
            z[n].copy_(fresh)
        ws.fill_(255)
        graph.replay()
        want = call(pa, "extend", z, max(new), cap, 0.1)
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
        for n in ("kpages", "vpages", "cpages"):
            assert torch.equal(y[n].view(torch.uint8), z[n].view(torch.uint8)), n
        y["cached"] += counts
        z["cached"] += counts


@pytest.mark.parametrize("new", [[2, 1, 5], [100, 3, 64]])
def test_results_do_not_depend_on_workspace_or_stream(gpu, new):
    """The same call again, on another stream with a workspace full of NaN: the same bits."""
    torch, pa = gpu
    x = pm.batch([500, 1500, 20], new, 2, 1, 128, 32, "bf16", True, seed=6)
    y = to_gpu(torch, x)
    first = call(pa, "attn", y, max(new), 1500, 0.1)
    ws = torch.full((pa.path_paged_workspace_bytes(3, sum(new), max(new), 1500, 2, 1, 128, pa.PATH_BF16),), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        again = call(pa, "attn", y, max(new), 1500, 0.1, workspace=ws)
    third = call(pa, "attn", y, max(new), 1500, 0.1, stream=stream, workspace=ws)
    torch.cuda.synchronize()
    for a, b, c in zip(first, again, third):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_a_prompt_in_chunks_then_tokens(gpu, oracle):
    """The calls as a server makes them: a prompt of 300 tokens in chunks of 130, drafts looked at and dropped, then single tokens -- against the
    library's own forward of the whole sequence, and the caches against its key prefill."""
    torch, pa = gpu
    H, d, L, page = 2, 64, 308, 32
    gen = torch.Generator().manual_seed(1)
    rn = lambda *s: torch.randn(*s, generator=gen)
    q, k, v = (rn(L, H, d) for _ in range(3))
    w, beta = torch.nn.functional.normalize(rn(L, H, d), dim=-1), 2 * torch.sigmoid(rn(L, H))
    x = {n: t.cuda() for n, t in dict(q=q, k=k, v=v, w=w, beta=beta).items()}
    kp, vp = torch.zeros(12, H, page, d, device="cuda"), torch.zeros(12, H, page, d, device="cuda")
    table = torch.tensor([[7, 0, 3, 11, 5, 1, 9, 2, 4, 8]], dtype=torch.int32, device="cuda")
    cached = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, at = [], 0
    for m in (130, 130, 40, 1, 1, 1, 4, 1):
        part = {n: t[at:at + m].contiguous() for n, t in x.items()}
        cu = torch.tensor([0, m], dtype=torch.int32, device="cuda")
        cache = (kp, vp, table, cached, cu, m, at)
        if m == 4:      # drafts: attention, then the append of the accepted ones, here all
            o, lse = pa.path_paged_attn(part["q"], part["k"], part["v"], part["w"], part["beta"], *cache)
            pa.path_paged_append(part["k"], part["v"], part["w"], part["beta"], *cache)
        else:
            o, lse = pa.path_paged_extend(part["q"], part["k"], part["v"], part["w"], part["beta"], *cache)
        out.append((o, lse))
        cached += m
        at += m
    heads = lambda t: t[:at].transpose(0, 1).contiguous()[None]
    ws = torch.empty(pa.path_attn_workspace_bytes(1, H, at, d, pa.PATH_F32), dtype=torch.uint8, device="cuda")
    want, wlse = pa.path_attn_fwd(heads(x["q"]), heads(x["k"]), heads(x["v"]), heads(x["w"]), heads(x["beta"]), workspace=ws)
    kc, vc = torch.zeros(1, H, at, d, device="cuda"), torch.zeros(1, H, at, d, device="cuda")
    pa.path_key_prefill(heads(x["v"]), ws, kc, vc)
    torch.cuda.synchronize()
    o, lse = torch.cat([a for a, _ in out]), torch.cat([b for _, b in out])
    assert (o - want[0].transpose(0, 1)).abs().max() <= 1e-4
    assert (lse - wlse[0].transpose(0, 1)).abs().max() <= 1e-4
    pos = torch.arange(at, device="cuda")
    mine = table[0].long()[pos // page]
    assert (kp[mine, :, pos % page] - kc[0].transpose(0, 1)).abs().max() <= 1e-4
    assert torch.equal(vp[mine, :, pos % page], vc[0].transpose(0, 1))


def test_far_pages(gpu):
    """Pages more than 4 GB into the pool."""
    torch, pa = gpu
    H, d, page = 8, 128, 256
    pool = 9000      # 4.7 GB each
    x = pm.batch([600], [3], H, 1, d, page, "bf16", seed=8, spare=0)
    y = to_gpu(torch, x)
    far = {n: torch.zeros(pool, H, page, d, dtype=torch.bfloat16, device="cuda") for n in ("kpages", "vpages")}
    where = torch.tensor([[8999, 8500, 4]], dtype=torch.int32)
    for i in range(3):
        for n in far:
            far[n][where[0, i]] = y[n][x["page_table"][0, i].long()]
    small = call(pa, "extend", y, 3, 600, 0.1)
    y2 = {**y, **far, "page_table": where.cuda()}
    big = call(pa, "extend", y2, 3, 600, 0.1)
    torch.cuda.synchronize()
    assert torch.equal(small[0], big[0]) and torch.equal(small[1], big[1])
    for i in range(3):
        for n in far:
            assert torch.equal(far[n][where[0, i]].view(torch.uint8), y[n][x["page_table"][0, i].long()].view(torch.uint8))


def test_a_call_while_another_device_is_current(gpu):
    torch, pa = gpu
    if torch.cuda.device_count() < 2:
        pytest.skip("one GPU")
    x = pm.batch([50], [2], 1, 1, 64, 16, "bf16", seed=1)
    y = to_gpu(torch, x)
    want = call(pa, "attn", y, 2, 50, 0.1)
    with torch.cuda.device(1):
        got = call(pa, "attn", y, 2, 50, 0.1)
    torch.cuda.synchronize(0)
    assert torch.equal(got[0], want[0])


def test_binding_refuses_tensors_of_another_kind(gpu):
    torch, pa = gpu
    y = to_gpu(torch, pm.batch([20], [3], 2, 1, 64, 16, "bf16", True))
    names = ("q", "k", "v", "w", "beta", "kpages", "vpages", "page_table", "cached", "cu_new")
    run = lambda **k: pa.path_paged_attn(*[{**y, **k}[n] for n in names], 3, 20, log_f=k.get("log_f", y["log_f"]), cpages=k.get("cpages", y["cpages"]),
                                         o=k.get("o"), lse=k.get("lse"), workspace=k.get("workspace"))
    run()
    for n in ("q", "v", "w", "beta", "kpages", "vpages", "log_f"):
        with pytest.raises(ValueError):
            run(**{n: y[n].float()})
        with pytest.raises(ValueError):
            run(**{n: y[n][..., :-1]})
        with pytest.raises(ValueError):
            run(**{n: y[n].cpu()})
    with pytest.raises(ValueError):
        run(w=y["w"].transpose(0, 1).contiguous().transpose(0, 1))
    for n in ("page_table", "cached", "cu_new"):
        with pytest.raises(ValueError):
            run(**{n: y[n].long()})
    with pytest.raises(ValueError):
        run(cached=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        run(cpages=None)
    with pytest.raises(ValueError):
        run(o=torch.empty_like(y["q"])[:2])
    with pytest.raises(pa.PathAttnError) as e:
        run(workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
    assert e.value.code in (1, 5)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("op", ["attn", "extend"])
@pytest.mark.parametrize("old,new", [([33], [1]), ([1100], [3]), ([500], [1]), ([700], [90])])
def test_infinite_values_stay_in_their_component(gpu, op, dtype, old, new):
    """An infinite value in the cache makes its own component infinite and leaves the others' bits alone."""
    torch, pa = gpu
    x = pm.batch(old, new, 2, 1, 64, 32, dtype, seed=12)
    y, z = to_gpu(torch, x), to_gpu(torch, x)
    n = old[0]
    for comp, row in ((5, n - 1), (9, n // 2), (11, 0)):
        z["vpages"][z["page_table"][0, row // 32].long(), :, row % 32, comp] = math.inf
    want, want_l = call(pa, op, y, new[0], n, 0.125)
    got, got_l = call(pa, op, z, new[0], n, 0.125)
    torch.cuda.synchronize()
    assert torch.equal(got_l, want_l) and torch.isfinite(want).all()
    rest = [i for i in range(64) if i not in (5, 9, 11)]
    assert torch.equal(got[..., rest], want[..., rest])
    assert (got[..., [5, 9, 11]] == math.inf).all()


def test_the_same_call_from_two_threads(gpu):
    """Two host threads, each with its own stream, workspace and cache."""
    import threading
    torch, pa = gpu
    x = pm.batch([300, 40], [70, 2], 2, 1, 64, 16, "bf16", True, seed=13)
    want_y = to_gpu(torch, x)
    want = call(pa, "extend", want_y, 70, 300, 0.1)
    torch.cuda.synchronize()
    got = [None, None]

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            y = to_gpu(torch, x)
            out = call(pa, "extend", y, 70, 300, 0.1)
        stream.synchronize()
        got[i] = (*out, y["kpages"])

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for o, lse, kp in got:
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1]) and torch.equal(kp.view(torch.uint8), want_y["kpages"].view(torch.uint8))


@pytest.mark.parametrize("seed", range(24))
def test_random_batches(gpu, seed):
    """Batches of up to nine sequences with lengths from nothing to several tiles, pages, groups, widths, types and gates at random."""
    import random
    r = random.Random(seed)
    S = r.choice([1, 1, 2, 3, 5, 9])
    old = [r.choice([0, 1, r.randint(2, 40), r.randint(41, 900)]) for _ in range(S)]
    new = [r.choice([0, 1, 1, r.randint(2, 16), r.randint(17, 64), r.randint(65, 200)]) for _ in range(S)]
    if not any(new):
        new[0] = 1
    G = r.choice([1, 1, 2, 3, 4, 7, 16])
    check(gpu, r.choice(["attn", "append", "extend", "extend"]), old, new, r.choice([1, 2, 3]), G, r.choice([64, 128]), r.choice([16, 32, 64, 128, 1024]),
          r.choice(["bf16", "bf16", "fp32"]), r.random() < 0.5, seed=100 + seed)


def test_many_short_sequences(gpu):
    """More sequences than a wave has lanes, some without new tokens, few and many new tokens mixed."""
    old = [(7 * i) % 90 for i in range(150)]
    new = [0 if i % 5 == 3 else 40 if i % 29 == 7 else 1 + i % 3 for i in range(150)]
    check(gpu, "extend", old, new, 2, 1, 64, 16, "bf16", True, seed=21)
    check(gpu, "attn", old, new, 1, 2, 64, 16, "fp32", False, seed=22)
