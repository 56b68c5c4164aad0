"""The append is linear in the keys, so keys a power of two larger or smaller must leave exactly so much larger or smaller caches, whichever way the
tokens go: nothing in between may have a narrower range than the keys' own type.  No tolerance."""
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


def append(pa, y, max_new, max_cached):
    pa.path_paged_append(*[y[n] for n in ("k", "v", "w", "beta", "kpages", "vpages", "page_table", "cached", "cu_new")], max_new, max_cached)


@pytest.mark.parametrize("power", [-60, -26, -17, 12, 17, 60])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [[1, 3], [40, 2], [150, 70]])
def test_keys_of_any_size_are_carried_alike(gpu, new, d, dtype, power):
    torch, pa = gpu
    old = [300, 77]
    x = pm.batch(old, new, 2, 1, d, 32, dtype, seed=31, unused=0.0)
    for n in ("k", "kpages"):      # elements below 2^-12 would leave the type's normal numbers at the lowest power before their products do
        x[n] = torch.where(x[n].abs() < 2.0 ** -12, torch.zeros_like(x[n]), x[n])
    y = {n: t.cuda() if t is not None else None for n, t in x.items()}
    z = {**y, "k": y["k"] * 2.0 ** power, "kpages": y["kpages"] * 2.0 ** power, "vpages": y["vpages"].clone()}
    y["kpages"] = y["kpages"].clone()
    before = y["kpages"].clone()
    append(pa, y, max(new), max(old))
    append(pa, z, max(new), max(old))
    torch.cuda.synchronize()
    assert not torch.equal(y["kpages"], before) and torch.isfinite(y["kpages"]).all()
    assert torch.equal(z["kpages"], y["kpages"] * 2.0 ** power), (z["kpages"].double() * 2.0 ** -power - y["kpages"].double()).abs().max()
