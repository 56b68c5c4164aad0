"""Memory that a paged call makes for itself when it is given a stream (run with -m gpu): it is that stream's own, so that no work pending on the caller's
stream can still use it, and it goes back to that stream."""
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


def stream_of(torch, t):
    """The stream whose memory t lies in, by the allocator's own record."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not in the allocator's memory")


def attn(pa, y, **more):
    return pa.path_paged_attn(*[y[n] for n in ("q", "k", "v", "w", "beta", "kpages", "vpages", "page_table", "cached", "cu_new")], 40, 300, **more)


@pytest.mark.parametrize("kind", ["stream", "handle"])
def test_made_tensors_are_of_the_given_stream(gpu, kind):
    torch, pa = gpu
    y = {n: t.cuda() if t is not None else None for n, t in pm.batch([300, 40], [40, 2], 2, 1, 64, 16, "bf16", seed=3).items()}
    want = attn(pa, y)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    o, lse = attn(pa, y, stream=s if kind == "stream" else s.cuda_stream)
    torch.cuda.synchronize()
    assert stream_of(torch, o) == s.cuda_stream and stream_of(torch, lse) == s.cuda_stream
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("kind", ["stream", "handle"])
def test_pending_work_on_freed_memory_does_not_reach_the_call(gpu, kind):
    """Blocks of the sizes that the call needs, freed on the current stream while their last fills are still queued there."""
    torch, pa = gpu
    y = {n: t.cuda() if t is not None else None for n, t in pm.batch([300, 40], [40, 2], 2, 1, 64, 16, "bf16", seed=3).items()}
    want = attn(pa, y)
    need = pa.path_paged_workspace_bytes(2, 42, 40, 300, 2, 1, 64, pa.PATH_BF16)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(50_000_000)      # (some tens of milliseconds: the fills wait behind it)
    junk = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (need, want[0].numel() * 2, want[1].numel() * 4)]
    for t in junk:
        t.fill_(255)
    del junk, t
    got = attn(pa, y, stream=s if kind == "stream" else s.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_given_tensors_stay_the_callers(gpu):
    """o given, lse made; the default stream by its handle, 0."""
    torch, pa = gpu
    y = {n: t.cuda() if t is not None else None for n, t in pm.batch([300], [4], 2, 1, 64, 16, "bf16", seed=3).items()}
    want = attn(pa, y)
    o = torch.empty_like(y["q"])
    torch.cuda.synchronize()
    for stream in (torch.cuda.Stream(), 0):
        got = attn(pa, y, o=o, stream=stream)
        torch.cuda.synchronize()
        assert got[0] is o and torch.equal(o, want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("kind", ["stream", "handle", "forked"])
def test_made_tensors_in_a_captured_call(gpu, kind):
    """The call given its stream while that is being captured, or another one forked from it, with everything made by the call: replayed between eager calls."""
    torch, pa = gpu
    y = {n: t.cuda() if t is not None else None for n, t in pm.batch([300, 40], [40, 2], 2, 1, 64, 16, "bf16", seed=3).items()}
    z = {n: t.cuda() if t is not None else None for n, t in pm.batch([300, 40], [40, 2], 2, 1, 64, 16, "bf16", seed=3).items()}
    s, other = torch.cuda.Stream(), torch.cuda.Stream()
    attn(pa, z)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        if kind == "forked":
            other.wait_stream(s)
        o, lse = attn(pa, y, stream={"stream": s, "handle": s.cuda_stream, "forked": other}[kind])
        if kind == "forked":
            s.wait_stream(other)
    for step in range(3):
        y["q"].copy_(torch.roll(z["q"], step, 0))
        graph.replay()
        want = attn(pa, {**z, "q": torch.roll(z["q"], step, 0)})
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1]), step
