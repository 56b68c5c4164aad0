"""What a new token's key and value hold shows in no row before it, also where they are infinities or NaN, on both ways and in every place of a tile of 64
(run with -m gpu).  Rows up to the token keep their log-sum-exp to the bit; their outputs stay within the bar of test_gpu_paged.py (the sum over a tile may be taken
in another order).  Bar on o: bf16 two half steps of max|v|, 2 * 2^-8 * max|v|; fp32 1e-4."""
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


def call(pa, op, y, max_new, max_cached):
    f = pa.path_paged_attn if op == "attn" else pa.path_paged_extend
    return f(*[y[n] for n in ("q", "k", "v", "w", "beta", "kpages", "vpages", "page_table", "cached", "cu_new")], max_new, max_cached, log_f=y["log_f"], cpages=y["cpages"])


@pytest.mark.parametrize("op", ["attn", "extend"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("old,new,at", [(37, 9, 3), (37, 9, 8), (0, 16, 15), (90, 100, 0), (90, 100, 31), (0, 100, 32), (700, 100, 63), (90, 100, 64), (90, 100, 77), (0, 100, 99),
                                        (90, 130, 129)])
def test_values_of_later_tokens_never_show(gpu, old, new, at, d, dtype, op):
    torch, pa = gpu
    x = pm.batch([old, 20], [new, 18], 2, 2, d, 32, dtype, gates=d == 64, seed=41)
    y = {n: t.cuda() if t is not None else None for n, t in x.items()}
    fresh = lambda **more: {**y, **{n: y[n].clone() for n in ("kpages", "vpages", "cpages") if y[n] is not None}, **more}
    want, want_l = call(pa, op, fresh(), max(new, 18), max(old, 20))
    v = y["v"].clone()
    v[at, :, 5], v[at, :, 11], v[at, 0, 40] = math.inf, -math.inf, math.nan
    got, got_l = call(pa, op, fresh(v=v), max(new, 18), max(old, 20))
    torch.cuda.synchronize()
    assert torch.equal(got_l, want_l) and torch.isfinite(want).all()
    bar = 1e-4 if dtype == "fp32" else 2 ** -7 * float(x["v"].abs().max())
    before = [t for t in range(new + 18) if t < at or t >= new]
    assert torch.isfinite(got[before]).all()
    assert (got[before].double() - want[before].double()).abs().max() <= bar
    for t in range(at, new):      # from the token on: its components, and no others
        rest = [i for i in range(d) if i not in (5, 11, 40)]
        assert (got[t, :, 5] == math.inf).all() and (got[t, :, 11] == -math.inf).all() and got[t, :2, 40].isnan().all(), t
        assert (got[t][:, rest].double() - want[t][:, rest].double()).abs().max() <= bar, t
        assert torch.isfinite(got[t, 2:, 40]).all()


@pytest.mark.parametrize("op", ["attn", "extend"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("old,new,at", [(37, 9, 4), (90, 100, 31), (0, 100, 70), (90, 100, 99)])
def test_keys_of_later_tokens_never_show(gpu, old, new, at, dtype, op):
    torch, pa = gpu
    x = pm.batch([old, 20], [new, 18], 2, 1, 64, 32, dtype, seed=42)
    y = {n: t.cuda() if t is not None else None for n, t in x.items()}
    fresh = lambda **more: {**y, **{n: y[n].clone() for n in ("kpages", "vpages")}, **more}
    want, want_l = call(pa, op, fresh(), max(new, 18), max(old, 20))
    for bad in (math.inf, math.nan):
        k = y["k"].clone()
        k[at, :, 7] = bad
        got, got_l = call(pa, op, fresh(k=k), max(new, 18), max(old, 20))
        torch.cuda.synchronize()
        before = [t for t in range(new + 18) if t < at or t >= new]
        assert torch.equal(got[before], want[before]) and torch.equal(got_l[before], want_l[before])
