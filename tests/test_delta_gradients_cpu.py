"""path_delta_train_bwd without a GPU: gradients that the caller brings are looked at as every other tensor is, and a workspace that is not there is named."""
import pytest
import torch

import delta_model as dm
import paper_2505_16381_amd as pa


def test_gradients_and_workspace_are_looked_at():
    x = dm.batch([5, 3], 2, 2, 64)
    ins = [x[n] for n in ("q", "k", "v", "beta", "d_o")]
    how = dict(log_f=x["log_f"], cu_seqlens=x["cu"], max_len=5, state_in=x["state"])
    ws = torch.empty(256, dtype=torch.uint8)
    with pytest.raises(ValueError, match="workspace"):
        pa.path_delta_train_bwd(*ins, None, **how)
    for name, bad in (("dq", x["v"]), ("dk", x["q"].float()), ("dv", x["q"]), ("dbeta", x["beta"][:, :2]), ("dlog_f", x["log_f"].float()), ("d_state_in", x["state"].bfloat16())):
        with pytest.raises(ValueError, match=f"{name} is"):
            pa.path_delta_train_bwd(*ins, ws, **how, **{name: bad})
    with pytest.raises(ValueError, match="goes with"):
        pa.path_delta_train_bwd(*ins, ws, **{**how, "log_f": None}, dlog_f=torch.empty_like(x["beta"]))
    with pytest.raises(ValueError, match="goes with"):
        pa.path_delta_train_bwd(*ins, ws, **{**how, "state_in": None}, d_state_in=torch.empty_like(x["state"]))
    with pytest.raises(ValueError, match="GPU"):
        pa.path_delta_train_bwd(*ins, ws, **how, dq=torch.empty_like(x["q"]))


def test_an_empty_step_needs_no_tokens():
    """T = 0: pointers to tokens may be NULL, for served calls too; what they carry on has to be there."""
    import ctypes
    at = 0x1000      # never read
    call = lambda tokens, o, states=at, T=0: pa.load_library().path_delta_extend(*[tokens] * 4, tokens, states, at, at, at, o, 2, T, 10, 4, 2, 1, 64, ctypes.c_float(0.1), 1, at, 1 << 40, None)
    assert call(None, None) == 0 and call(at, at) == 0
    assert call(None, None, states=None) == 1
    assert call(at, None, T=20) == 1 and call(None, at, T=20) == 1
