"""Host bounds of the paged calls that do not fit 32 bits are refused, not cut to their low bits."""
import pytest
import torch

import paged_model as pm
import paper_2505_16381_amd as pa


def test_workspace_of_bounds_past_32_bits_is_refused():
    good = [2, 100, 64, 3000, 4, 2, 128]
    assert pa.path_paged_workspace_bytes(*good, pa.PATH_BF16) > 0
    for i in range(7):
        for x in (good[i] + (1 << 32), good[i] - (1 << 32), 1 << 31):
            assert pa.path_paged_workspace_bytes(*good[:i], x, *good[i + 1:], pa.PATH_BF16) == 0, (i, x)


@pytest.mark.parametrize("max_new,max_cached", [((1 << 32) + 3, 20), (3, (1 << 32) + 20), (-(1 << 32) + 3, 20), (3, 1 << 31)])
def test_calls_with_bounds_past_32_bits_are_refused(monkeypatch, max_new, max_cached):
    """(tensors on the CPU that say they are on a GPU; the library is not to be reached)"""
    x = pm.batch([20], [3], 2, 1, 64, 16, "bf16")
    args = [x[n] for n in ("q", "k", "v", "w", "beta", "kpages", "vpages", "page_table", "cached", "cu_new")]
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    class Library:
        def __getattr__(self, name):
            raise AssertionError(f"{name} reached")

    monkeypatch.setattr(pa.binding, "load_library", Library)
    ws = torch.empty(1 << 20, dtype=torch.uint8)
    for call in (lambda **k: pa.path_paged_attn(*args, **k), lambda **k: pa.path_paged_extend(*args, **k), lambda **k: pa.path_paged_append(*args[1:], **k)):
        with pytest.raises(ValueError, match="32-bit"):
            call(max_new=max_new, max_cached=max_cached, workspace=ws)
