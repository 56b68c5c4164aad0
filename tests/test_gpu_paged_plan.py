"""Page tables made on the GPU against lists (delta_model.plan): whole numbers, equal."""
import random

import pytest

import delta_model as dm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    import paper_2505_16381_amd as pa
    assert torch.cuda.is_available()
    pa.load_library()
    return torch, pa


def check(gpu, cached, new, table, free, count, T, page, **more):
    torch, pa = gpu
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    t, f, c = ints(table), ints(free), ints([count])
    ws = torch.full((pa.path_paged_plan_workspace_bytes(len(table), len(table[0]), T),), 255, dtype=torch.uint8, device="cuda")
    cu, slots, missing = pa.path_paged_plan(ints(cached), ints(new), t, f, c, T, page, workspace=ws, **more)
    torch.cuda.synchronize()
    want = dm.plan(cached, new, table, free, count, T, page)
    assert slots.dtype == torch.int64
    got = (t.tolist(), f.tolist(), c.item(), cu.tolist(), slots.tolist(), missing.tolist())
    for name, a, b in zip(("table", "free", "count", "cu", "slots", "missing"), got, want):
        assert a == b, name
    return got


def server(rng, nseq, P, page, pool, turns, gpu, most=60):
    """A server's turns: sequences go on, drop drafts, end and begin."""
    table, free, count = [[-1] * P for _ in range(nseq)], rng.sample(range(pool), pool), pool
    lengths = [0] * nseq
    for _ in range(turns):
        cached = [0 if rng.random() < 0.2 else max(0, n - rng.randint(0, 5)) for n in lengths]
        new = [rng.choice([0, 1, 1, rng.randint(0, most)]) for _ in range(nseq)]
        T = sum(new) + rng.choice([0, 0, 3])
        table, free, count, *_ = check(gpu, cached, new, table, free, count, T, page)
        lengths = [min(a + b, P * page) for a, b in zip(cached, new)]


@pytest.mark.parametrize("nseq,P,page,pool", [(1, 1, 16, 1), (1, 5, 16, 9), (3, 4, 32, 12), (70, 9, 16, 300), (5, 64, 16, 400), (63, 130, 16, 5000), (200, 65, 64, 6000), (1100, 3, 16, 2000)])
def test_servers(gpu, nseq, P, page, pool):
    server(random.Random(nseq + P), nseq, P, page, pool, 6, gpu)


@pytest.mark.parametrize("nseq,P,pool", [(4, 10, 7), (200, 64, 900)])
def test_pool_used_up(gpu, nseq, P, pool):
    rng = random.Random(1)
    server(rng, nseq, P, 16, pool, 5, gpu, most=P * 16)


@pytest.mark.parametrize("nseq,P", [(3, 6), (130, 70)])
def test_entries_that_are_no_pages(gpu, nseq, P):
    """Entries outside the pool are holes: replaced where new tokens come, kept under cached ones, dropped behind; a full stack drops what is given back; counts outside the stack are held to it."""
    rng = random.Random(3)
    pool = nseq * P
    pages = rng.sample(range(pool), pool)
    table = [[pages.pop() if rng.random() < 0.6 else rng.choice([-1, -7, pool, 1 << 30, -(1 << 31)]) for _ in range(P)] for _ in range(nseq)]
    for count in (len(pages), pool, 0, -4, pool + 5, 1 << 30):
        free = pages + [0] * (pool - len(pages))
        cached = [rng.randint(-3, P * 16 + 20) for _ in range(nseq)]
        new = [rng.randint(-5, 90) for _ in range(nseq)]
        check(gpu, cached, new, table, free, count, sum(max(0, m) for m in new), 16)


def test_offsets_end_at_the_bound(gpu):
    check(gpu, [0, 3, 9], [10, 20, 30], [[-1] * 4] * 3, list(range(12)), 12, 25, 16)
    check(gpu, [0, 3, 9], [10, 20, 30], [[-1] * 4] * 3, list(range(12)), 12, 0, 16)
    check(gpu, [0] * 5, [0x7fffffff] * 5, [[-1] * 4] * 5, list(range(9)), 9, 100, 16)
    check(gpu, [0x7fffffff, 0], [5, 0x7fffffff], [[-1] * 4] * 2, list(range(9)), 9, 1000, 4096)


def test_many_tokens(gpu):
    """Prompts of tens of thousands of tokens beside single ones."""
    rng = random.Random(9)
    new = [rng.choice([1, rng.randint(1, 30000)]) for _ in range(40)]
    check(gpu, [rng.randint(0, 5000) for _ in new], new, [[-1] * 200 for _ in new], rng.sample(range(9000), 9000), 9000, sum(new), 256)


def test_captured(gpu):
    """One captured call follows lengths and tables through its replays."""
    torch, pa = gpu
    for nseq, P in ((6, 20), (300, 40)):
        rng = random.Random(nseq)
        pool, page, T = nseq * P // 2, 16, nseq * 40
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        table, free, count = [[-1] * P for _ in range(nseq)], list(range(pool)), pool
        t, f, c, cached, new = ints(table), ints(free), ints([count]), ints([0] * nseq), ints([0] * nseq)
        ws = torch.empty(pa.path_paged_plan_workspace_bytes(nseq, P, T), dtype=torch.uint8, device="cuda")
        pa.path_paged_plan(cached, new, t, f, c, T, page, workspace=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = pa.path_paged_plan(cached, new, t, f, c, T, page, workspace=ws)
        for _ in range(4):
            a, b = [rng.randint(0, P * page) for _ in range(nseq)], [rng.randint(0, 40) for _ in range(nseq)]
            cached.copy_(ints(a))
            new.copy_(ints(b))
            g.replay()
            torch.cuda.synchronize()
            table, free, count, *rest = dm.plan(a, b, table, free, count, T, page)
            assert (t.tolist(), f.tolist(), c.item()) == (table, free, count)
            assert [x.tolist() for x in out] == rest
            torch.randn(1 << 20, device="cuda").sum().item()      # (the program's own work)
