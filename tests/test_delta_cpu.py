"""Gated delta rule and page tables without a GPU: refusals come before anything is launched, a workspace covers every smaller problem, and the models of the GPU tests
agree with differences and with each other's plain forms."""
import ctypes
import random

import pytest
import torch

import delta_model as dm
import paper_2505_16381_amd as pa

F = ctypes.c_float
Z = 0x1000      # never read: every case below fails before


def forward(name="path_delta_fwd", ptr=None, nseq=2, T=200, L=100, H=2, G=1, d=64, layout=0, scale=0.1, dt=1, ws=Z, wsb=1 << 40):
    p = [Z] * 9
    p[5] = None      # no offsets: sequences of one length
    for i, v in (ptr or {}).items():
        p[i] = v
    return getattr(pa.load_library(), name)(*p, nseq, T, L, H, G, d, layout, F(scale), dt, ws, wsb, None)


def backward(ptr=None, nseq=2, T=200, L=100, H=2, G=1, d=64, layout=0, scale=0.1, dt=1, ws=Z, wsb=1 << 40):
    p = [Z] * 15
    p[5] = None
    for i, v in (ptr or {}).items():
        p[i] = v
    return pa.load_library().path_delta_train_bwd(*p, nseq, T, L, H, G, d, layout, F(scale), dt, ws, wsb, None)


def extend(ptr=None, nseq=2, T=20, L=10, slots=4, H=2, G=1, d=64, scale=0.1, dt=1, ws=Z, wsb=1 << 40):
    p = [Z] * 10
    for i, v in (ptr or {}).items():
        p[i] = v
    return pa.load_library().path_delta_extend(*p, nseq, T, L, slots, H, G, d, F(scale), dt, ws, wsb, None)


def plan(ptr=None, nseq=2, T=20, pool=40, page=16, per=10, ws=Z, wsb=1 << 40):
    p = [Z] * 8
    for i, v in (ptr or {}).items():
        p[i] = v
    return pa.load_library().path_paged_plan(*p, nseq, T, pool, page, per, ws, wsb, None)


@pytest.mark.parametrize("name", ["path_delta_fwd", "path_delta_train_fwd"])
def test_forward_refuses_before_it_launches(name):
    call = lambda **k: forward(name, **k)
    for i in (0, 1, 2, 3, 7):
        assert call(ptr={i: None}) == 1, i
    assert call(ws=None) == 1
    assert call(dt=4) == 3
    for bad in (dict(nseq=0), dict(T=-1), dict(L=0), dict(H=0), dict(G=0), dict(d=96), dict(d=32), dict(T=201), dict(H=70000), dict(H=40000, G=2),
                dict(nseq=1 << 20, T=1 << 20, L=1, H=2), dict(nseq=(1 << 18) + 1, T=(1 << 18) + 1, L=1, H=2), dict(nseq=1, T=1 << 28, L=1 << 28, H=2)):
        assert call(**bad) == 2, bad
    assert call(scale=0.0) == 4 and call(scale=float("nan")) == 4 and call(layout=2) == 4
    assert call(ptr={5: Z}) == 4      # a packed batch is [T, heads, d]
    assert call(wsb=256) == 5 and call(ws=Z + 16) == 5
    for i in (0, 1, 2, 6, 7, 8):
        assert call(ptr={i: Z + 8}) == 7, i


def test_backward_refuses_before_it_launches():
    for i in (0, 1, 2, 3, 7, 9, 10, 11, 12):
        assert backward(ptr={i: None}) == 1, i
    for i in (4, 13, 6, 14):      # gates and their gradients, states and theirs go together
        assert backward(ptr={i: None}) == 1, i
    assert backward(dt=3) == 3
    for bad in (dict(nseq=0), dict(d=100), dict(T=3), dict(G=0)):
        assert backward(**bad) == 2, bad
    assert backward(layout=5) == 4
    assert backward(wsb=0) == 5 and backward(ws=Z + 128) == 5
    for i in (0, 1, 2, 6, 7, 8, 9, 10, 11, 14):
        assert backward(ptr={i: Z + 4}) == 7, i


def test_extend_refuses_before_it_launches():
    for i in (0, 1, 2, 3, 5, 6, 7, 8, 9):
        assert extend(ptr={i: None}) == 1, i
    assert extend(dt=9) == 3
    for bad in (dict(nseq=0), dict(T=-5), dict(L=0), dict(slots=0), dict(d=48), dict(H=-1)):
        assert extend(**bad) == 2, bad
    assert extend(scale=-1.0) == 4
    assert extend(wsb=8) == 5
    for i in (0, 1, 2, 5, 9):
        assert extend(ptr={i: Z + 2}) == 7, i
    assert extend(T=0) == 0      # nothing to do


def test_plan_refuses_before_it_launches():
    for i in range(8):
        assert plan(ptr={i: None}) == 1, i
    assert plan(ws=None) == 1
    for bad in (dict(nseq=0), dict(T=-1), dict(pool=0), dict(per=0), dict(page=8), dict(page=48), dict(page=8192), dict(page=0), dict(nseq=(1 << 22) + 1)):
        assert plan(**bad) == 2, bad
    assert plan(wsb=4) == 5 and plan(ws=Z + 4) == 5


def test_workspaces_cover_every_smaller_problem():
    rng = random.Random(5)
    for _ in range(300):
        big = [rng.randint(1, 40), rng.randint(0, 20000), rng.randint(1, 5000), rng.randint(1, 12), rng.randint(1, 4), rng.choice([64, 128])]
        small = [rng.randint(1, big[0]), rng.randint(0, big[1]), rng.randint(1, big[2]), rng.randint(1, big[3]), rng.randint(1, big[4]), rng.choice([64, big[5]])]
        for dt in (0, 1):
            for training in (False, True):
                assert 0 < pa.path_delta_workspace_bytes(*small, dt, training) <= pa.path_delta_workspace_bytes(*big, dt, training)
            assert pa.path_delta_workspace_bytes(*big, dt) <= pa.path_delta_workspace_bytes(*big, dt, True)
    assert pa.path_delta_workspace_bytes(1, 100, 100, 1, 1, 96, 1) == 0 and pa.path_delta_workspace_bytes(1, 1 << 32, 100, 1, 1, 64, 1) == 0
    assert pa.path_delta_workspace_bytes(1, 100, 100, 1, 1, 64, 3) == 0
    assert 0 < pa.path_paged_plan_workspace_bytes(3, 10, 5) <= pa.path_paged_plan_workspace_bytes(4, 10, 5)
    assert pa.path_paged_plan_workspace_bytes(0, 10, 5) == 0 and pa.path_paged_plan_workspace_bytes(1 << 32, 10, 5) == 0


def test_binding_refuses():
    x = dm.batch([5, 3], 2, 2, 64)
    qkvb = (x["q"], x["k"], x["v"], x["beta"])
    with pytest.raises(ValueError, match="max_len"):
        pa.path_delta_fwd(*qkvb, cu_seqlens=x["cu"])
    with pytest.raises(ValueError, match="packed"):
        pa.path_delta_fwd(*[t[None] for t in qkvb], cu_seqlens=x["cu"], max_len=5)
    with pytest.raises(ValueError, match="32-bit"):
        pa.path_delta_fwd(*qkvb, cu_seqlens=x["cu"], max_len=1 << 40)
    with pytest.raises(ValueError, match="layout"):
        pa.path_delta_fwd(*[t[None] for t in qkvb], layout=3)
    with pytest.raises(ValueError, match="multiple"):
        pa.path_delta_fwd(x["v"][:, :3], x["v"][:, :3], x["v"], x["beta"], cu_seqlens=x["cu"], max_len=5)
    with pytest.raises(ValueError, match="GPU"):
        pa.path_delta_fwd(*qkvb, cu_seqlens=x["cu"], max_len=5)      # (tensors of the CPU)
    with pytest.raises(ValueError, match="workspace"):
        pa.path_delta_train_fwd(*qkvb, cu_seqlens=x["cu"], max_len=5)
    with pytest.raises(ValueError, match="states"):
        pa.path_delta_extend(*qkvb, x["state"][0], torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), x["cu"], 5)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    with pytest.raises(ValueError, match="page_table"):
        pa.path_paged_plan(i32(2), i32(2), i32(2), i32(4), i32(1), 3, 16)
    with pytest.raises(ValueError, match="32-bit"):
        pa.path_paged_plan(i32(2), i32(2), i32(2, 3), i32(4), i32(1), 1 << 31, 16)
    with pytest.raises(ValueError, match="GPU"):
        pa.path_paged_plan(i32(2), i32(2), i32(2, 3), i32(4), i32(1), 3, 16)


def test_model_gradients_against_differences():
    """Every gradient of the model's reverse recurrence against central differences, in random directions."""
    x = dm.batch([7, 0, 4], 2, 2, 8, "fp32", seed=3)
    x = {n: t.double() if t is not None and t.is_floating_point() else t for n, t in x.items()}
    scale = 0.37
    loss = lambda y, st: sum(float((a * b).nansum()) for a, b in zip(dm.forward(y, scale, st), (x["d_o"], x["d_state"])))
    grads = dict(zip(("q", "k", "v", "beta", "log_f", "state"), dm.backward(x, scale, x["state"], x["d_state"])))
    g = torch.Generator().manual_seed(1)
    for n, want in grads.items():
        for _ in range(3):
            w = torch.randn(x[n].shape, generator=g, dtype=torch.float64)
            h = 1e-5
            up, down = (loss({**x, n: x[n] + e * w}, x["state"] + e * w if n == "state" else x["state"]) for e in (h, -h))
            got, exact = (up - down) / (2 * h), float((want * w).sum())
            assert abs(got - exact) <= 1e-6 * max(1.0, abs(exact)), (n, got, exact)      # (h^2 and 1e-16 / h)


def test_chunk_form_is_the_recurrence():
    """The formulas that the kernels evaluate, by chunks of any size, against the token walk: outputs, states and gradients."""
    x = dm.batch([23], 1, 1, 8, "fp32", seed=9)
    q, k, v, beta, log_f, d_o = (x[n][:, 0].double() for n in ("q", "k", "v", "beta", "log_f", "d_o"))
    scale = 0.6
    o, last = dm.forward(x, scale, x["state"])
    want = dm.backward(x, scale, x["state"], x["d_state"])
    for C in (1, 5, 8, 23):
        S, G = x["state"][0, 0].double(), x["d_state"][0, 0].double()
        kept, got = [], [torch.zeros_like(t) for t in (q, k, v, beta, log_f)]
        for c in range(0, 23, C):
            sl = slice(c, min(c + C, 23))
            K, Q, V, be, b = k[sl], q[sl], v[sl], beta[sl], torch.cumsum(log_f[sl], 0)
            gamma, rho = torch.exp(b), torch.exp(b[-1] - b)
            D = torch.exp(b[:, None] - b).tril()
            L, M = (D * (K @ K.T)).tril(-1), scale * D * (Q @ K.T)
            eye = torch.eye(len(b), dtype=torch.float64)
            P = torch.linalg.inv(eye + L * be)
            E = P @ (V - gamma[:, None] * (K @ S))
            U = be[:, None] * E
            assert torch.allclose(scale * gamma[:, None] * (Q @ S) + M @ U, o[sl, 0], atol=1e-12)
            kept.append((sl, S, E, U, P, L, M, D, gamma, rho))
            S = gamma[-1] * S + K.T @ (rho[:, None] * U)
        assert torch.allclose(S, last[0, 0], atol=1e-12)
        for sl, S0, E, U, P, L, M, D, gamma, rho in reversed(kept):
            K, Q, be, dO = k[sl], q[sl], beta[sl], d_o[sl]
            A = torch.eye(len(be), dtype=torch.float64) - be[:, None] * (P @ L)
            Y = A.T @ (M.T @ dO + rho[:, None] * (K @ G))
            X, N = Y @ U.T, dO @ U.T
            Gq, Gk = scale * (N * D).tril(), -(be[:, None] * X * D).tril(-1)
            dq = Gq @ K + scale * gamma[:, None] * (dO @ S0.T)
            read = Gk @ K - (gamma * be)[:, None] * (Y @ S0.T)
            UG = rho[:, None] * (U @ G.T)
            written = Gk.T @ K + Gq.T @ Q + UG
            sums = (Q * dq).sum(1) + (K * (read - written)).sum(1)
            got[0][sl], got[1][sl], got[2][sl], got[3][sl] = dq, read + written, be[:, None] * Y, (Y * E).sum(1)
            got[4][sl] = torch.flip(torch.cumsum(torch.flip(sums, [0]), 0), [0]) + gamma[-1] * (S0 * G).sum() + (K * UG).sum()
            G = gamma[-1] * G + Q.T @ (scale * gamma[:, None] * dO) - K.T @ ((gamma * be)[:, None] * Y)
        for a, w in zip((*got, G), want):
            assert torch.allclose(a, w.reshape(a.shape), atol=1e-11)


def test_plan_model_keeps_every_page():
    """Random servers: no page is lost or in two places, tokens of a sequence that misses nothing have slots of their own."""
    rng = random.Random(7)
    for trial in range(30):
        nseq, P, page, pool = rng.randint(1, 6), rng.randint(1, 8), 16, rng.randint(1, 40)
        table, free, count = [[-1] * P for _ in range(nseq)], list(range(pool)), pool
        for _ in range(12):
            cached, new = [rng.choice([0, rng.randint(0, P * page)]) for _ in range(nseq)], [rng.choice([0, 1, rng.randint(0, 60)]) for _ in range(nseq)]
            table, free, count, cu, slots, missing = dm.plan(cached, new, table, free, count, sum(new), page)
            held = [e for r in table for e in r if e >= 0]
            assert sorted(held + free[:count]) == list(range(pool))
            given = [x for x in slots if x >= 0]
            assert len(set(given)) == len(given)
            if not any(missing):
                assert all(-1 not in r[-(-c // page):min(P, -(-(c + m) // page))] for r, c, m in zip(table, cached, new))
