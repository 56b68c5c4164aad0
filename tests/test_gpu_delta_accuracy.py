"""Gated delta rule on the GPU: values of unlike sizes within a head, against the token walk in 64 bits.  Bars as in test_gpu_delta.py, which derives them."""
import pytest

import delta_model as dm
from test_gpu_delta import close, poison, to_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    import paper_2505_16381_amd as pa
    assert torch.cuda.is_available()
    pa.load_library()
    return torch, pa


def pair(gpu, x, d, H, G, dtype="bf16", state=True):
    """o, last states, gradients of the training pair on the inputs x, and the same of the walk."""
    torch, pa = gpu
    y, scale, L = to_gpu(x), d ** -0.5, max(b - a for a, b in zip(x["cu"].tolist(), x["cu"].tolist()[1:]))
    ins = [y[n] for n in ("q", "k", "v", "beta")]
    how = dict(log_f=y["log_f"], scale=scale, cu_seqlens=y["cu"], max_len=L, workspace=poison(torch, pa, x, H, G, d, L, dtype, True), state_in=y["state"] if state else None)
    out = pa.path_delta_train_fwd(*ins, final_state=state, **how)
    got = dict(zip(("o", "state") if state else ("o",), out if state else (out,)))
    names = ["dq", "dk", "dv", "dbeta"] + (["dlog_f"] if x["log_f"] is not None else []) + (["d_state"] if state else [])
    got.update(zip(names, pa.path_delta_train_bwd(*ins, y["d_o"], d_state_out=y["d_state"] if state else None, **how)))
    first = x["state"] if state else None
    want = dict(zip(("o", "state"), dm.forward(x, scale, first)))
    want.update(zip(("dq", "dk", "dv", "dbeta", "dlog_f", "d_state"), dm.backward(x, scale, first, x["d_state"] if state else None)))
    return got, {n: want[n] for n in got}


@pytest.mark.parametrize("down", [22, 28])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("G", [1, 2])
def test_small_columns_of_a_head(gpu, down, d, dtype, G):
    """Sixteen value indices 2^-22 and 2^-28 below the rest of their head: what belongs to a value index (o, states, dv) is right to the bars by these columns' own size."""
    torch, pa = gpu
    x = dm.batch([130, 40], 2, G, d, dtype, seed=11)
    for n in ("v", "d_o", "state", "d_state"):
        x[n][..., 16:32] *= 2.0 ** -down
    got, want = pair(gpu, x, d, 2, G, dtype)
    for n in ("o", "dv", "state", "d_state"):
        for part in (slice(0, 16), slice(16, 32), slice(32, d)):
            close(torch, n, got[n][..., part], want[n][..., part], x["cu"].tolist(), dtype == "fp32")
    for n in ("dq", "dk", "dbeta", "dlog_f"):
        close(torch, n, got[n], want[n], x["cu"].tolist(), dtype == "fp32")
