"""The paged calls' binding names the tensor whose axes are in another order than the kernels read, also where its number of elements is the same (every
other entry point of the library takes heads first, so that is the mistake to expect)."""
import pytest
import torch

import paged_model as pm
import paper_2505_16381_amd as pa

NAMES = ("q", "k", "v", "w", "beta", "kpages", "vpages", "page_table", "cached", "cu_new")


def calls(x, **more):
    y = {**x, **more}
    gates = dict(log_f=y["log_f"], cpages=y["cpages"])
    out = {n: y[n] for n in ("o", "lse") if n in y}
    args = [y[n] for n in NAMES]
    return [lambda: pa.path_paged_attn(*args, 3, 20, **gates, **out), lambda: pa.path_paged_extend(*args, 3, 20, **gates, **out),
            lambda: pa.path_paged_append(*args[1:], 3, 20, **gates)]


def head_major(x):
    """(name, the tensor with its first two axes exchanged, contiguous)"""
    y = {**x, "o": torch.empty_like(x["q"]), "lse": torch.empty(x["q"].shape[:2], device=x["q"].device)}
    return [(n, y[n].transpose(0, 1).contiguous()) for n in ("v", "w", "beta", "log_f", "kpages", "vpages", "cpages", "o", "lse")]


def refused_by_name(x):
    for name, t in head_major(x):
        for call in calls(x, **{name: t})[:2 if name in ("o", "lse") else 3]:
            with pytest.raises(ValueError, match=rf"\b{'k' if name == 'kpages' else name}"):
                call()
    for name in ("cached", "cu_new"):
        for call in calls(x, **{name: x[name][:, None].contiguous()}):
            with pytest.raises(ValueError, match=rf"^{name} is"):
                call()


def test_other_orders_of_axes_are_refused_by_name():
    refused_by_name(pm.batch([20], [3], 2, 1, 64, 16, "bf16", True))


@pytest.mark.gpu
def test_other_orders_of_axes_are_refused_on_the_gpu():
    assert torch.cuda.is_available()
    x = {n: t.cuda() for n, t in pm.batch([20], [3], 2, 1, 64, 16, "bf16", True).items()}
    for call in calls(x):
        call()      # (as they are: accepted)
    torch.cuda.synchronize()
    refused_by_name(x)
