"""Bounds that would need a launch of 2^32 threads or more, which HIP does not take, are refused before anything is launched -- a call that fails at its last launch
has already written new keys -- and bounds just below are not.  (No GPU: the pointers are never read.)"""
import ctypes

import pytest

import paper_2505_16381_amd as pa

Z = 0x1000
BASE = dict(nseq=1, T=64, max_new=64, max_cached=4096, H=1, G=1, d=64)
# (what is too large, bounds, the bound to halve, dt: 0 fp32, 1 bf16)
TOO_LARGE = [
    ("rows to join, fp32", dict(T=1 << 20, max_new=1 << 20, G=64), "T", 0),
    ("sweep over the new tokens", dict(T=1 << 22, max_new=1 << 22, G=64), "T", 1),
    ("pieces of a chunk's cache", dict(nseq=65535, T=100, max_new=100, max_cached=300000), "nseq", 1),
    ("keys carried on", dict(nseq=1024, H=32, T=4096, max_new=100, max_cached=1 << 21), "max_cached", 1),
    ("keys carried on, fp32", dict(nseq=1024, H=32, T=4096, max_new=100, max_cached=1 << 21), "max_cached", 0),
]


def bounds(more):
    b = {**BASE, **more}
    return b, 4096, -(-max(b["max_cached"], 1) // 4096)


def call(name, more, dt):
    b, page, per = bounds(more)
    lib = pa.load_library()
    lengths = [b["nseq"], b["T"], b["max_new"], b["max_cached"], 8, page, per, b["H"]]
    if name == "path_paged_append":
        p = [Z] * 11
        p[4] = p[7] = None
        return lib.path_paged_append(*p, *lengths, b["d"], dt, Z, 1 << 62, None)
    p = [Z] * 14
    p[5] = p[8] = None
    return getattr(lib, name)(*p, *lengths, b["G"], b["d"], ctypes.c_float(0.1), dt, Z, 1 << 62, None)


def workspace(more, dt):
    b, _, _ = bounds(more)
    return pa.path_paged_workspace_bytes(*[b[n] for n in ("nseq", "T", "max_new", "max_cached", "H", "G", "d")], dt)


@pytest.mark.parametrize("what,more,halve,dt", TOO_LARGE, ids=lambda x: x.replace(" ", "_") if isinstance(x, str) else "")
def test_launches_past_32_bits_are_refused_first(what, more, halve, dt):
    assert workspace(more, dt) == 0
    for name in ("path_paged_attn", "path_paged_extend", "path_paged_append"):
        if name != "path_paged_append" or more.get("G", 1) == 1:
            assert call(name, more, dt) == 2, name
    assert workspace({**more, halve: more[halve] // 2}, dt) > 0
