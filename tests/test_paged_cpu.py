"""Paged caches without a GPU: refusals come before anything is launched, the workspace covers every smaller problem, and the 64-bit model of the
GPU tests agrees with the decode oracle, with which it shares nothing."""
import ctypes
import random

import numpy as np
import pytest
import torch

import paged_model as pm
import paper_2505_16381_amd as pa
from oracle import decode_oracle as dec

F = ctypes.c_float
Z = 0x1000      # never read: every case below fails before


def attn(name="path_paged_attn", ptr=None, nseq=2, T=8, max_new=4, max_cached=100, num_pages=40, page=16, per=10, H=2, G=1, d=64, scale=0.1, dt=1, ws=Z, wsb=1 << 40):
    p = [Z] * 14
    for i, v in (ptr or {}).items():
        p[i] = v
    return getattr(pa.load_library(), name)(*p, nseq, T, max_new, max_cached, num_pages, page, per, H, G, d, F(scale), dt, ws, wsb, None)


def append(ptr=None, nseq=2, T=8, max_new=4, max_cached=100, num_pages=40, page=16, per=10, H=2, d=64, dt=1, ws=Z, wsb=1 << 40):
    p = [Z] * 11
    for i, v in (ptr or {}).items():
        p[i] = v
    return pa.load_library().path_paged_append(*p, nseq, T, max_new, max_cached, num_pages, page, per, H, d, dt, ws, wsb, None)


@pytest.mark.parametrize("name", ["path_paged_attn", "path_paged_extend"])
def test_attention_refuses_before_it_launches(name):
    call = lambda **k: attn(name, **k)
    for i in (0, 1, 2, 3, 4, 6, 7, 9, 10, 11, 12, 13):
        assert call(ptr={i: None}) == 1, i
    assert call(ptr={5: None}) == 1 and call(ptr={8: None}) == 1      # gates without sums, sums without gates
    assert call(ws=None) == 1
    assert call(dt=5) == 3
    for bad in (dict(nseq=0), dict(T=-1), dict(max_new=0), dict(max_cached=-1), dict(H=0), dict(G=0), dict(G=65), dict(d=96), dict(d=32), dict(num_pages=0),
                dict(per=0), dict(page=8), dict(page=48), dict(page=8192), dict(page=0), dict(max_cached=161), dict(nseq=40000, H=2), dict(T=1 << 29),
                dict(H=2000, G=64)):
        assert call(**bad) == 2, bad
    assert call(scale=0.0) == 4 and call(scale=-1.0) == 4 and call(scale=float("nan")) == 4
    assert call(wsb=64) == 5 and call(ws=Z + 16) == 5
    for i in (0, 1, 2, 3, 6, 7, 8, 12):
        assert call(ptr={i: Z + 8}) == 7, i
    assert call(T=0) == 0      # nothing to do


def test_append_refuses_before_it_launches():
    for i in (0, 1, 2, 3, 5, 6, 8, 9, 10):
        assert append(ptr={i: None}) == 1, i
    assert append(ptr={4: None}) == 1 and append(ptr={7: None}) == 1
    assert append(dt=2) == 3
    for bad in (dict(nseq=0), dict(max_new=0), dict(d=100), dict(page=24), dict(max_cached=1000)):
        assert append(**bad) == 2, bad
    assert append(wsb=8) == 5 and append(ws=Z + 1) == 5
    for i in (0, 1, 2, 5, 6, 7):
        assert append(ptr={i: Z + 4}) == 7, i
    assert append(T=0) == 0


def test_workspace_bytes():
    wb = lambda nseq=2, T=100, max_new=64, max_cached=3000, H=4, G=2, d=128, dt=1: pa.path_paged_workspace_bytes(nseq, T, max_new, max_cached, H, G, d, dt)
    assert wb() > 0 and wb() % 256 == 0
    for bad in (dict(nseq=0), dict(d=96), dict(dt=3), dict(G=65), dict(max_new=0), dict(T=-1)):
        assert wb(**bad) == 0, bad
    assert wb(T=0) > 0
    assert wb(T=1, max_new=1, nseq=1) < 1 << 20      # one token: records only
    lib = pa.load_library()
    for T, max_new, max_cached in ((1, 1, 5), (8, 4, 90), (500, 300, 5000), (700, 16, 0)):      # a call takes what was said, and not a byte less
        n = pa.path_paged_workspace_bytes(3, T, max_new, max_cached, 2, 1, 64, 0)
        assert attn(nseq=3, T=T, max_new=max_new, max_cached=max_cached, per=400, dt=0, wsb=n - 1) == 5
        assert append(nseq=3, T=T, max_new=max_new, max_cached=max_cached, per=400, dt=0, wsb=64 if n > 64 else 0) == 5


def test_workspace_of_larger_bounds_serves_smaller_calls():
    """A server keeps one workspace, made for its largest call."""
    rng = random.Random(5)
    for case in range(20000):
        big = [rng.choice(r) for r in ((1, 2, 5, 16, 64, 300), (1, 16, 17, 100, 255, 256, 700, 5000), (1, 4, 16, 17, 600, 5000),
                                       (0, 100, 700, 5000, 70000, 1 << 20), (1, 2, 7, 16, 40, 128), (1, 2, 3, 4, 16, 17, 64), (64, 128))]
        small = [x if rng.random() < .5 else rng.randint(min(x, low), x) for x, low in zip(big, (1, 0, 1, 0, 1, 1, 64))]
        small[6] = 64 if small[6] < 128 else 128
        dt = rng.randrange(2)
        need, have = pa.path_paged_workspace_bytes(*small, dt), pa.path_paged_workspace_bytes(*big, dt)
        assert need <= have or have == 0, (small, big, dt)      # (0: the larger bounds are rejected)


def test_binding_refuses_what_the_kernels_would_misread():
    x = pm.batch([5], [2], 2, 1, 64, 16, "fp32")
    args = lambda **k: [{**x, **k}[n] for n in ("q", "k", "v", "w", "beta", "kpages", "vpages", "page_table", "cached", "cu_new")]
    with pytest.raises(ValueError, match="GPU"):      # tensors on the CPU
        pa.path_paged_attn(*args(), 2, 5)
    with pytest.raises(ValueError):
        pa.path_paged_attn(*args(k=x["k"][0]), 2, 5)
    with pytest.raises(TypeError):
        pa.path_paged_attn(*args(k=x["k"].half()), 2, 5)


@pytest.mark.parametrize("gates", [False, True])
def test_model_agrees_with_the_decode_oracle(gates):
    """Chunks of the model, token by token of the oracle: o, lse and the caches."""
    H, d, page = 2, 64, 16
    for old, new in (([20], [5]), ([0], [3]), ([33, 1], [1, 7])):
        x = pm.batch(old, new, H, 1, d, page, "fp32", gates, seed=sum(old))
        o, lse, kp, vp, cp = pm.expect(x, 0.1, "extend")
        for s, n in enumerate(old):
            m, t0 = new[s], int(x["cu_new"][s])
            pages, slots = pm.rows_of(x, s, n)
            get = lambda t: t[pages, :, slots].transpose(0, 1).double().numpy()
            kc, vc = get(x["kpages"]), get(x["vpages"])
            cc = x["cpages"].double()[pages, :, slots].T.numpy() if gates else None
            for t in range(t0, t0 + m):
                a = [x[i][t].double().numpy() for i in ("q", "k", "v", "w", "beta")]
                got = dec.decode_step(*a, kc, vc, 0.1, None, *((x["log_f"][t].double().numpy(), cc) if gates else ()))
                np.testing.assert_allclose(o[t], got[0], atol=1e-12)
                np.testing.assert_allclose(lse[t], got[1], atol=1e-12)
                kc, vc = got[2], got[3]
                cc = got[4] if gates else None
            pages, slots = pm.rows_of(x, s, n + m)
            np.testing.assert_allclose(kp[pages, :, slots].transpose(0, 1), kc, atol=1e-12)
            np.testing.assert_allclose(vp[pages, :, slots].transpose(0, 1), vc, atol=1e-12)
            if gates:
                np.testing.assert_allclose(cp[pages, :, slots].T, cc, atol=1e-12)
