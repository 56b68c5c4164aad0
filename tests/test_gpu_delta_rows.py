"""Rows that belong to no sequence are left as they are: in o, and in every gradient that the caller brings.  Bars as in test_gpu_delta.py."""
import pytest

import delta_model as dm
from test_gpu_delta import close, to_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    import paper_2505_16381_amd as pa
    assert torch.cuda.is_available()
    pa.load_library()
    return torch, pa


@pytest.mark.parametrize("cu,max_len,true", [([0, 70, 79], 70, [0, 70, 79]),             # rows behind the last sequence
                                             ([10, 80, 129], 70, [10, 80, 129]),         # rows before the first one
                                             ([0, 90, 129], 66, [(0, 66), (90, 129)]),    # tokens past the bound on lengths
                                             ([0, 100, 20], 129, [(0, 100)])], ids=str)   # offsets that fall
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("G", [1, 2])
def test_rows_of_no_sequence_in_gradients(gpu, cu, max_len, true, d, dtype, G):
    torch, pa = gpu
    x = dm.batch([70, 9], 2, G, d, dtype, tail=50, seed=6)
    x["cu"] = torch.tensor(cu, dtype=torch.int32)
    y, f32 = to_gpu(x), dtype == "fp32"
    spans = true if isinstance(true[0], tuple) else list(zip(true, true[1:]))
    ins = [y[n] for n in ("q", "k", "v", "beta")]
    how = dict(log_f=y["log_f"], cu_seqlens=y["cu"], max_len=max_len,
               workspace=torch.full((pa.path_delta_workspace_bytes(2, 129, max_len, 2, G, d, 0 if f32 else 1, True),), 255, dtype=torch.uint8, device="cuda"))
    o = torch.full_like(y["v"], 7.0)
    assert pa.path_delta_train_fwd(*ins, o=o, **how) is o
    names = ["dq", "dk", "dv", "dbeta", "dlog_f"]
    mine = {n: torch.full_like(y[n[1:]], 7.0) for n in names}
    got = pa.path_delta_train_bwd(*ins, y["d_o"], **how, **mine)
    assert len(got) == 5 and all(a is mine[n] for a, n in zip(got, names))
    idle = torch.ones(129, dtype=torch.bool)
    for a, b in spans:
        idle[a:b] = False
    for n, t in dict(mine, o=o).items():
        assert idle.any() and (t[idle.cuda()] == 7.0).all(), n
    for a, b in spans:
        part = {n: t[a:b] if n in ("q", "k", "v", "beta", "log_f", "d_o") else t for n, t in x.items()}
        part["cu"] = torch.tensor([0, b - a])
        want = dict(zip(("dq", "dk", "dv", "dbeta", "dlog_f"), dm.backward(part, d ** -0.5)), o=dm.forward(part, d ** -0.5)[0])
        for n, t in dict(mine, o=o).items():
            close(torch, n, t[a:b], want[n], [0, b - a], f32)


def test_state_gradients_of_the_caller(gpu):
    torch, pa = gpu
    y = to_gpu(dm.batch([40, 80], 2, 1, 64))
    ins = [y[n] for n in ("q", "k", "v", "beta")]
    how = dict(log_f=y["log_f"], cu_seqlens=y["cu"], max_len=80, state_in=y["state"], workspace=torch.empty(pa.path_delta_workspace_bytes(2, 120, 80, 2, 1, 64, 1, True), dtype=torch.uint8, device="cuda"))
    pa.path_delta_train_fwd(*ins, **how)
    want = pa.path_delta_train_bwd(*ins, y["d_o"], d_state_out=y["d_state"], **how)
    mine = torch.full_like(y["state"], 7.0)
    got = pa.path_delta_train_bwd(*ins, y["d_o"], d_state_out=y["d_state"], d_state_in=mine, **how)
    assert len(got) == 6 and got[-1] is mine and all(torch.equal(a, b) for a, b in zip(got, want))
