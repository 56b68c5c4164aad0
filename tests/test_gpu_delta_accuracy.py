"""Gated delta rule on the GPU: values of unlike sizes within a head, against the token walk in 64 bits.  Bars as in test_gpu_delta.py, which derives them."""
import math

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


def wide_betas(torch, x):
    """beta = 2 sigmoid(N(2, 1)), as the attention's own inputs have it: half of all above 1.76."""
    g = torch.Generator().manual_seed(5)
    x["beta"] = (2 * torch.sigmoid(2 + torch.randn(x["beta"].shape, generator=g))).to(x["q"].dtype)


def keys_alike(torch, x, part):
    """Unit keys and queries whose products are `part` on average."""
    g = torch.Generator().manual_seed(6)
    m = torch.nn.functional.normalize(torch.randn(1, *x["k"].shape[1:], generator=g), dim=-1)
    for n in ("q", "k"):
        x[n] = torch.nn.functional.normalize(part ** 0.5 * m + (1 - part) ** 0.5 * x[n].float(), dim=-1).to(x["v"].dtype)


@pytest.mark.parametrize("alike", [0.0, 0.7, 0.95])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("state", [True, False])
def test_wide_betas_and_keys_alike(gpu, alike, d, state):
    """Sums that cancel: betas near 2 over keys that resemble each other, no gates.  Bars on the root mean square of a head's error, beside what rounding the exact result once to bf16 makes of it (the two
    are independent, their squares add up; a per cent for the draw of 4e4 values and more):
      o               sums of products of operands of 22 bits; rows of P add up to 66 at most (two equal keys, beta 2, add 2 |E| a step), so 66 * 2^-22 * sqrt(8): 4.5e-5 of the norm, half of 1e-4.
      dv              Y, kept as one fp16 number: at most 2^-11, over a binade 0.58 * 0.7 of that in deviation, 2e-4; and o's: 3e-4 at most.
      dq, dk, dbeta   up to eight such roundings: 8e-4."""
    torch, pa = gpu
    x = dm.batch([640], 2, 1, d, seed=3)
    wide_betas(torch, x)
    x["log_f"][:] = 0
    if alike:
        keys_alike(torch, x, alike)
    got, want = pair(gpu, x, d, 2, 1, state=state)
    for n, bar in (("o", 1e-4), ("dv", 3e-4), ("dq", 8e-4), ("dk", 8e-4), ("dbeta", 8e-4)):
        for h in range(2):
            a, w = got[n][:, h].double().cpu(), want[n][:, h]
            size = float(w.square().mean())
            off, least = float((a - w).square().mean()) / size, float((w.bfloat16().double() - w).square().mean()) / size
            assert off <= 1.01 ** 2 * least + bar ** 2, (n, h, off ** 0.5, least ** 0.5)


@pytest.mark.parametrize("d", [64, 128])
def test_outputs_do_not_depend_on_whether_states_are_wanted(gpu, d):
    """The same bits of o, from the forward and the training forward, with the last states handed out or not; also where the state is 3000 times the values that come in."""
    torch, pa = gpu
    from test_gpu_delta import pushes_one_way
    x = dm.batch([1500, 70], 2, 1, d, seed=1)
    pushes_one_way(torch, x)
    k = torch.zeros(d)
    k[: d // 4] = (d // 4) ** -0.5 if d == 64 else 0.17578125      # 16 of 1/4: of length one; 32 of 45/256: 0.9944
    x["k"][:], x["q"][:] = k.bfloat16(), k.bfloat16()
    for z in (dm.batch([130, 1, 700], 2, 2, d, seed=4), x):
        y, G = to_gpu(z), z["v"].shape[1] // 2
        ins, L = [y[n] for n in ("q", "k", "v", "beta")], 1500
        how = dict(log_f=y["log_f"], cu_seqlens=y["cu"], max_len=L)
        ws = lambda: poison(torch, pa, z, 2, G, d, L, "bf16", True)
        o, _ = pa.path_delta_train_fwd(*ins, final_state=True, workspace=ws(), **how)
        close(torch, "o", o, dm.forward(z, d ** -0.5)[0], z["cu"].tolist(), False)
        for other in (pa.path_delta_train_fwd(*ins, workspace=ws(), **how), pa.path_delta_fwd(*ins, **how), pa.path_delta_fwd(*ins, final_state=True, **how)[0]):
            assert torch.equal(other, o)


def gate_gradients(torch, x, head, rounded):
    """dlog_f of a value head of one sequence whose length is a multiple of 64, by the chunks' formulas in 64 bits; `rounded`: what the chunks' gradients start from -- the state before, the gradient behind,
    E and Y -- rounded to fp16 (over 2^-4: values of size one, as over their power of two)."""
    G, d = x["v"].shape[1] // x["q"].shape[1], x["v"].shape[2]
    q, k = (x[n][:, head // G].double() for n in ("q", "k"))
    v, beta, log_f, d_o = (x[n][:, head].double() for n in ("v", "beta", "log_f", "d_o"))
    kept = (lambda t: (16 * t).half().double() / 16) if rounded else (lambda t: t)
    S, g, chunks, eye, out = torch.zeros(d, d).double(), torch.zeros(d, d).double(), [], torch.eye(64).double(), torch.zeros_like(beta)
    for c in range(0, len(q), 64):
        sl = slice(c, c + 64)
        K, b = k[sl], torch.cumsum(log_f[sl], 0)
        D = torch.exp(b[:, None] - b).tril()
        L, M = (D * (K @ K.T)).tril(-1), d ** -0.5 * D * (q[sl] @ K.T)
        P = torch.linalg.inv(eye + L * beta[sl])
        E = P @ (v[sl] - torch.exp(b)[:, None] * (K @ S))
        chunks.append((sl, b, D, L, M, P, S, E))
        S = torch.exp(b[-1]) * S + K.T @ (torch.exp(b[-1] - b)[:, None] * (beta[sl, None] * E))
    for sl, b, D, L, M, P, S, E in reversed(chunks):
        K, Q, be, dO, gamma, rho = k[sl], q[sl], beta[sl, None], d_o[sl], torch.exp(b)[:, None], torch.exp(b[-1] - b)[:, None]
        Y = (eye - be * (P @ L)).T @ (M.T @ dO + rho * (K @ g))
        Sr, gr, Er, Yr = kept(S), kept(g), kept(E), kept(Y)
        Gq, Gk = d ** -0.5 * (dO @ (be * Er).T * D).tril(), -(be * (Yr @ (be * Er).T) * D).tril(-1)
        dq, read, UG = Gq @ K + d ** -0.5 * gamma * (dO @ Sr.T), Gk @ K - gamma * be * (Yr @ Sr.T), rho * (be * Er) @ gr.T
        sums = (Q * dq).sum(1) + (K * (read - Gk.T @ K - Gq.T @ Q - UG)).sum(1)
        out[sl] = torch.flip(torch.cumsum(torch.flip(sums, [0]), 0), [0]) + gamma[-1] * (Sr * gr).sum() + (K * UG).sum()
        g = gamma[-1] * g + Q.T @ (d ** -0.5 * gamma * dO) - K.T @ (gamma * be * Y)
    return out


@pytest.mark.parametrize("beta", [1, 2])
@pytest.mark.parametrize("alike", [0.7, 0.95])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 2])
def test_gradients_of_gates_over_keys_alike(gpu, beta, alike, d, G):
    """dlog_f adds up Gq_ri (q_r . k_i) and Gk_ri (k_r . k_i) over the pairs i < t <= r of a chunk.  Over keys alike all products are near one and the pairs' weights cancel, so an independent error of each weight
    does not: 2^-12 of them left 6e-3 of the result.  The bar: what rounding the state, its gradient, E and Y to single fp16 numbers, the only ones that are, makes of the result in 64 bits; 1.5 times that for another draw
    of some 640 roundings and what two-part operands add (they are 2^11 times better), beside the result's own rounding and a tenth of it."""
    torch, pa = gpu
    x = dm.batch([640], 2, G, d, seed=3)
    if beta == 2:
        wide_betas(torch, x)
    x["log_f"][:] = 0
    keys_alike(torch, x, alike)
    got, want = pair(gpu, x, d, 2, G, state=False)
    for h in range(2 * G):
        a, w = got["dlog_f"][:, h].double().cpu(), want["dlog_f"][:, h]
        assert (gate_gradients(torch, x, h, False) - w).abs().max() <= 1e-10 * w.abs().max()
        size = float(w.square().mean())
        off, least = float((a - w).square().mean()) / size, float((w.bfloat16().double() - w).square().mean()) / size
        kept = float((gate_gradients(torch, x, h, True) - w).square().mean()) / size
        assert off <= 1.1 ** 2 * least + 1.5 ** 2 * kept, (h, off ** 0.5, least ** 0.5, kept ** 0.5)


def largest_states(torch, x, scale):
    """The root mean square of each sequence's head's state, and of its gradient, where it is largest: [nseq,V,1,1] each."""
    kept, cu, rms = [], x["cu"].tolist(), lambda t: t.square().mean((-1, -2), keepdim=True).sqrt()
    dm.forward(x, scale, x["state"], kept)
    G = x["v"].shape[1] // x["q"].shape[1]
    q, k = (x[n].double().repeat_interleave(G, 1) for n in ("q", "k"))
    beta, f, d_o = x["beta"].double(), torch.exp(x["log_f"].double()), x["d_o"].double()
    states, grads = [], []
    for s, (a, b) in enumerate(zip(cu, cu[1:])):
        states.append(torch.stack([rms(t) for t in kept[a:b]]).amax(0))
        g, sizes = x["d_state"][s].double(), []
        for t in range(b - 1, a - 1, -1):
            sizes.append(rms(g))
            g = g + scale * q[t, :, :, None] * d_o[t, :, None]
            g = f[t, :, None, None] * (g - k[t, :, :, None] * (beta[t, :, None] * torch.einsum("hij,hi->hj", g, k[t]))[:, None])
        grads.append(torch.stack(sizes).amax(0))
    return torch.stack(states), torch.stack(grads)


@pytest.mark.parametrize("up,down,period", [(0.15, -0.16, 40), (0.3, -0.3, 14), (0.02, -0.02, 200), (0.43, -3.0, 8)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("G", [1, 2])
def test_gates_that_grow(gpu, up, down, period, d, dtype, G):
    """log_f above zero for a while, and below for as long, no run of tokens adding up to more than 3: states and gradients grow up to e^3 times (within seven tokens, or twenty) and fall again.  The bars are
    the usual ones; those of the states are relative to the largest that a head's state gets to in the sequence, for operands of two fp16 numbers end with fp16's smallest steps: an entry of P that has fallen
    to e^-3 is off by 2^-25 as one of size one is, and is multiplied with rows that hang on the state at its largest."""
    torch, pa = gpu
    x = dm.batch([200, 70], 2, G, d, dtype, seed=13)
    at = torch.arange(270)
    rises = at % period < period // 2 if down > -3 else at % period < period - 1
    x["log_f"][:] = torch.where(rises, up, down)[:, None].to(x["log_f"].dtype)
    x["log_f"][:, 1] = 0
    got, want = pair(gpu, x, d, 2, G, dtype)
    sizes = dict(zip(("state", "d_state"), largest_states(torch, x, d ** -0.5)))
    for n in got:
        if n in sizes and dtype == "bf16":
            off = (got[n].double().cpu() - want[n]).abs()
            assert (off <= (1e-5 if n == "state" else 2e-5) * sizes[n]).all(), (n, float((off / sizes[n]).max()))
        else:
            close(torch, n, got[n], want[n], x["cu"].tolist(), dtype == "fp32")


@pytest.mark.parametrize("up,down,period", [(0.45, -0.5, 40), (0.35, -0.36, 40), (1.4, -9.9, 8)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 2])
def test_gates_that_grow_far(gpu, up, down, period, d, G):
    """Runs of tokens within a chunk that add up to s = 7 to 9.8: gamma and rho alone would be past fp16's end as factors of operands.  o and the 16-bit gradients to the usual bars.  States, relative to the largest they get
    to: an entry of P or M is off by up to 2^-25 whatever its size, hence by 2^-25 e^s of one that a run as long has taken to e^-s, and its product with a row of what has grown e^s times by as much; a row adds up 64 of them
    in every chunk: sqrt(64) * 0.58 (the deviation), about 5."""
    torch, pa = gpu
    x = dm.batch([200, 70], 2, G, d, seed=13)
    at = torch.arange(270)
    saw = down > -3
    x["log_f"][:] = torch.where(at % period < (period // 2 if saw else period - 1), up, down)[:, None].to(x["log_f"].dtype)
    x["log_f"][:, 1] = 0
    s = up * (period // 2 if saw else period - 1)
    got, want = pair(gpu, x, d, 2, G)
    sizes = dict(zip(("state", "d_state"), largest_states(torch, x, d ** -0.5)))
    for n in got:
        if n in sizes:
            off = (got[n].double().cpu() - want[n]).abs()
            assert (off <= (5 * 2.0 ** -25 * math.exp(s) + 1e-5) * sizes[n]).all(), (n, float((off / sizes[n]).max()))
        else:
            close(torch, n, got[n], want[n], x["cu"].tolist(), False)
