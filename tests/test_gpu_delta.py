"""Gated delta rule on the GPU against the token walk in 64 bits (delta_model.py).

Bars, relative to the root mean square r of a sequence's head in the tensor (inputs: unit q and k, values of size one; e = half a step of bf16 = 2^-8,
h = half a step of fp16 = 2^-11, deviation h / sqrt(3) = 2.8e-4):
  o, dq, dk, dv (bf16)   the result is rounded once, e of it.  Before that it is a sum of products of rounded operands; from input to output a value passes up to eight such
                         roundings (state, prediction's error, P, U, M; backwards as many again), each 2.8e-4 of the sum's norm: sqrt(8) * 2.8e-4 = 8e-4 r, and the
                         largest of 1e5 values five deviations away, more where a token's own sum is above the mean: e |x| + 8e-3 r.
  dbeta, dlog_f (bf16)   dot products of d, and of d^2 and 64 d, such values, rounded once: as above, on tensors with longer tails: e |x| + 2e-2 r.
  states, d_state        fp32 accumulation of products of 23-bit operands: 2^-23 of the sum's norm each, five deviations of sqrt(8) of them 2e-6, and as much for
                         fp32 sums over 64 tokens a chunk: 1e-5 r.  (bf16 tensors, states handed out.)
  all of it (fp32)       sums of up to d and 64 terms in 32 bits, a triangular solve of 64 rows: sqrt(64 * 8) * 2^-24 = 1.3e-6 of the norm, five deviations: 1e-5 r; dot products
                         of d^2 terms (dlog_f) 4e-5 r.
r is of the token's own row where that is more than its sequence's: a row's error is a part of the norm of its own terms.  dv_r = beta_r (A^T dU)_r with dU = M^T dO + rho K G is of the
size of rho_r K_r G, and rho falls with the distance from the sequence's end, so with gates of mean 1/2 the last rows, next to d_state (values of size 0.3 * sqrt(d) = 3 in K_r G), are
ten times the mean over 130 tokens, and 1e-5 of the mean would be 1e-6 of them: less than the sqrt(512) * 2^-24 that one row's sums are given.
d_state (bf16) 2e-5 r: M = scale tril(D QK^T) in two parts of fp16 is off by up to 2^-25 whatever its size, for the lower part ends with fp16's smallest steps, and its entries are of the size
scale / sqrt(d) = 2^-6 here, so that is 2^-19 of them: more than the 2^-23 above.  It goes through dU = M^T dO and Y to sum K^T (gamma beta Y): half of 2^-25 in deviation (0.58 of it) times
sqrt(33) rows times values of size one is 1e-7 in Y; times K's 1/8, beta's 0.6 and the root of some 8 rows before gamma has fallen, 2.1e-8 in d_state, and 1e-7 at five deviations.  Heads
whose first gates fall fast have r near 0.01 (scale * 1/8 * gamma of size one, over few rows), so that is 1e-5 r from M alone, and as much again is the bar.
dbeta and dlog_f: r is the largest of the sequence's head where that is more than its mean.  dbeta_t = Y_t . E_t is a dot product of d terms off by its factors' errors, 2^-24 and up of
|Y_t| |E_t|, and the last token has |Y| = |K G| = 7.8 and |E| up to 9.8 where the mean of |Y| over 130 tokens is 0.18 (one key for all tokens, gates of mean 1/2): 61 * 2^-24 = 3.6e-6 beside a
mean dbeta of 0.21, of which 1e-5 is 2.1e-6.  Two rows of random values have |Y| |E| / sqrt(d) as their product, so the largest |dbeta| measures it.  dlog_f sums such products."""
import math
import random

import pytest

import delta_model as dm

pytestmark = pytest.mark.gpu

E16 = 2.0 ** -8


@pytest.fixture(scope="module")
def gpu():
    import torch
    import paper_2505_16381_amd as pa
    assert torch.cuda.is_available()
    pa.load_library()
    return torch, pa


def to_gpu(x):
    return {n: t.cuda() if t is not None else None for n, t in x.items()}


def close(torch, name, got, want, cu, f32, least=1e-30):
    """`want` [T,heads,..] or, of states, [nseq,V,d,d], 64 bits; sequence by sequence and head by head."""
    got, want = got.double().cpu(), want.double()
    rel, bar = (0.0, 4e-5 if name == "dlog_f" else 1e-5) if f32 or "state" in name else (E16, 2e-2 if name in ("dbeta", "dlog_f") else 8e-3)
    bar *= 1 if f32 or name != "d_state" else 2
    parts = [slice(a, b) for a, b in zip(cu[:-1], cu[1:])] if "state" not in name else range(len(want))
    for i, p in enumerate(parts):
        g, w = (got[p][None], want[p][None]) if "state" in name else (got[p], want[p])
        if g.numel() == 0:
            continue
        r = w.transpose(0, 1).flatten(1).square().mean(1).sqrt().view(1, -1, *[1] * (w.dim() - 2))
        if "state" not in name and w.dim() == 3:
            r = torch.maximum(r, w.square().mean(2, keepdim=True).sqrt())
        if name in ("dbeta", "dlog_f"):
            r = w.abs().amax(0, keepdim=True)
        off = float(((g - w).abs() - rel * w.abs() - bar * r).max())
        fits = off <= least      # (False for NaN)
        assert fits, (name, i, off, float((g - w).abs().max()), float(r.max()))


def laid(torch, t, B, layout):
    """A packed tensor of B sequences of one length as [B,heads,L,..] or [B,L,heads,..]."""
    t = t.view(B, -1, *t.shape[1:])
    return t.transpose(1, 2).contiguous() if layout == 0 else t.contiguous()


def flat(t, layout):
    return (t.transpose(1, 2) if layout == 0 else t).flatten(0, 1)


def poison(torch, pa, x, H, G, d, L, dtype, training):
    nseq = len(x["cu"]) - 1
    n = pa.path_delta_workspace_bytes(nseq, x["q"].shape[0], L, H, G, d, 1 if dtype == "bf16" else 0, training)
    return torch.full((n,), 255, dtype=torch.uint8, device="cuda")      # (NaN as fp16, fp32, bf16)


def train(gpu, lengths, H=2, G=1, d=64, dtype="bf16", gates=True, layout="packed", state=True, d_state=True, seed=0, tail=0, change=None, max_len=None, without=True, check=close):
    torch, pa = gpu
    x = dm.batch(lengths, H, G, d, dtype, gates, seed, tail=tail)
    if change:
        change(torch, x)
    y, scale, cu = to_gpu(x), d ** -0.5, x["cu"].tolist()
    L, names = max_len or max(1, max(lengths)), ["q", "k", "v", "beta", "log_f", "d_o"]
    ws = poison(torch, pa, x, H, G, d, L, dtype, True)
    how = dict(scale=scale, workspace=ws, state_in=y["state"] if state else None)
    if layout == "packed":
        how.update(cu_seqlens=y["cu"], max_len=L)
        z = y
    else:
        layout = dict(bhld=0, blhd=1)[layout]
        how.update(layout=layout)
        z = {n: laid(torch, y[n], len(lengths), layout) if y[n] is not None else None for n in names}
    back = (lambda t: t) if layout == "packed" else (lambda t: flat(t, layout))
    o, last = pa.path_delta_train_fwd(z["q"], z["k"], z["v"], z["beta"], log_f=z["log_f"], final_state=True, **how)
    got = pa.path_delta_train_bwd(z["q"], z["k"], z["v"], z["beta"], z["d_o"], log_f=z["log_f"], d_state_out=y["d_state"] if d_state else None, **how)
    again = pa.path_delta_train_bwd(z["q"], z["k"], z["v"], z["beta"], z["d_o"], log_f=z["log_f"], d_state_out=y["d_state"] if d_state else None, **how)
    assert all(torch.equal(a, b) for a, b in zip(got, again))      # from one workspace as often as wanted, the same bits
    how["workspace"] = poison(torch, pa, x, H, G, d, L, dtype, False)
    o1, last1 = pa.path_delta_fwd(z["q"], z["k"], z["v"], z["beta"], log_f=z["log_f"], final_state=True, **how)
    assert torch.equal(o1, o) and torch.equal(last1, last)
    o2 = o if not without else pa.path_delta_fwd(z["q"], z["k"], z["v"], z["beta"], log_f=z["log_f"], **how)      # no states wanted: operands of fewer parts
    want_o, want_last = dm.forward(x, scale, x["state"] if state else None)
    want = dm.backward(x, scale, x["state"] if state else None, x["d_state"] if d_state else None)
    f32 = dtype == "fp32"
    close(torch, "o", back(o), want_o, cu, f32)
    close(torch, "o", back(o2), want_o, cu, f32)
    check(torch, "state", last, want_last, cu, f32)
    out = ["dq", "dk", "dv", "dbeta"] + (["dlog_f"] if gates else []) + (["d_state"] if state else [])
    assert len(got) == len(out)
    full = dict(zip(("dq", "dk", "dv", "dbeta", "dlog_f", "d_state"), want))
    for n, t in zip(out, got):
        check(torch, n, t if n == "d_state" else back(t), full[n], cu, f32)
    return got


LENGTHS = [[1], [2], [15, 17], [63], [64], [65], [128, 1, 127], [0, 5, 0, 64, 0], [200, 129]]


@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_lengths(gpu, lengths, d, dtype):
    train(gpu, lengths, 2, 1, d, dtype, seed=len(lengths) + d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,G", [(1, 1), (3, 1), (1, 2), (2, 3), (5, 4)])
def test_heads(gpu, d, dtype, H, G):
    train(gpu, [70, 3, 130], H, G, d, dtype, seed=H * 10 + G)


@pytest.mark.parametrize("layout", ["bhld", "blhd"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("G", [1, 2])
def test_layouts(gpu, layout, d, dtype, G):
    train(gpu, [100, 100, 100], 2, G, d, dtype, layout=layout, seed=d + G)


@pytest.mark.parametrize("gates", [True, False])
@pytest.mark.parametrize("state", [True, False])
@pytest.mark.parametrize("d_state", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_without_gates_or_states(gpu, gates, state, d_state, dtype):
    train(gpu, [90, 130], 2, 2, 64, dtype, gates=gates, state=state, d_state=d_state, seed=4)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_no_tokens(gpu, dtype):
    """A packed batch of empty sequences hands its states on, and their gradients back."""
    torch, pa = gpu
    y = to_gpu(dm.batch([0, 0], 2, 2, 64, dtype))
    ins, how = [y[n] for n in ("q", "k", "v", "beta")], dict(log_f=y["log_f"], cu_seqlens=y["cu"], max_len=1)
    assert y["q"].numel() == 0
    o, last = pa.path_delta_fwd(*ins, state_in=y["state"], final_state=True, **how)
    assert o.shape == y["v"].shape and torch.equal(last, y["state"])
    assert (pa.path_delta_fwd(*ins, final_state=True, **how)[1] == 0).all() and pa.path_delta_fwd(*ins, **how).numel() == 0
    ws = torch.empty(pa.path_delta_workspace_bytes(2, 0, 1, 2, 2, 64, 1 if dtype == "bf16" else 0, True), dtype=torch.uint8, device="cuda")
    o, last = pa.path_delta_train_fwd(*ins, state_in=y["state"], final_state=True, workspace=ws, **how)
    got = pa.path_delta_train_bwd(*ins, y["d_o"], ws, state_in=y["state"], d_state_out=y["d_state"], **how)
    assert torch.equal(last, y["state"]) and torch.equal(got[-1], y["d_state"]) and all(t.numel() == 0 for t in got[:-1])
    assert all(t.numel() == 0 for t in pa.path_delta_train_bwd(*ins, y["d_o"], ws, **how))


@pytest.mark.parametrize("n", [64, 65, 300, 4200])
def test_many_sequences(gpu, n):
    """Chunks are found among as many sequences as there are: empty ones, short ones and some of several chunks."""
    rng = random.Random(n)
    lengths = [rng.choice([0, 0, 1, 2, 3]) for _ in range(n)]
    for i in (0, 63, n // 2, n - 1):
        lengths[i] = rng.choice([64, 65, 130])

    # dlog_f of a sequence of one token is what is left of gamma <S, G> and what the token reads and writes, of which the first is a sum of 4096 products of 0.3 by 1, each off by
    # 0.58 * sqrt(2) * 2^-12 (S and G as single fp16 numbers): 64 * 0.3 * 2e-4 = 3.8e-3 in deviation, 1.9e-2 at five of them, with as much from the others 2.7e-2.
    # dbeta of one is a single Y.E with |Y| = |K G| = 8 and |E| = 8.4: 67 / 8 * 2e-4 = 1.7e-3, five of them 8.4e-3.
    # fp32: 67 * 2^-24 for each factor; <S, G> is of the size of 64 * 0.3 = 19, off by 2^-24 of that for each of some 17 steps of its sum.
    def check(torch, name, got, want, cu, f32):
        close(torch, name, got, want, cu, f32, least={"dlog_f": 17 * 19 * 2 ** -24, "dbeta": 2 * 67 * 2 ** -24}.get(name, 1e-30) if f32 else {"dlog_f": 2.7e-2, "dbeta": 8.4e-3}.get(name, 1e-30))

    train(gpu, lengths, 1, 2, 64, seed=n, check=check)
    train(gpu, lengths, 1, 1, 64, "fp32", seed=n, check=check)


def test_many_workgroups(gpu):
    """Heads enough that a workgroup takes 32 columns (256 workgroups of them, and more)."""
    for d, dtype in ((64, "bf16"), (128, "bf16"), (64, "fp32")):
        train(gpu, [66] * 9, 4, 4, d, dtype, seed=2)


def gates_that_forget(torch, x):
    x["log_f"][3] = -math.inf
    x["log_f"][70] = -1e30
    x["log_f"][100:110] = -50.0


def gates_that_keep(torch, x):
    x["log_f"][:] = 0.0


def betas_at_the_ends(torch, x):
    x["beta"][::3] = 0.0
    x["beta"][1::3] = 1.0
    x["beta"][2::3] = 2.0


def betas_of_nothing(torch, x):
    x["beta"][:] = 0.0


def the_same_key(torch, x):
    x["k"][:] = x["k"][0]


def keys_in_turn(torch, x):
    x["k"][:] = x["k"][0]
    x["k"][1::2] *= -1


def empty_keys(torch, x):
    x["k"][5:60] = 0
    x["q"][8:50] = 0


def small(torch, x):
    for n in ("v", "d_o", "state", "d_state"):
        x[n] *= 2.0 ** -60


def large(torch, x):
    for n in ("v", "d_o", "state", "d_state"):
        x[n] *= 2.0 ** 40


def heads_of_all_sizes(torch, x):
    w = 2.0 ** torch.tensor([-30.0, 0.0, 25.0])
    for n in ("v", "d_o"):
        x[n] *= w[:, None].to(x[n].dtype)
    for n in ("state", "d_state"):
        x[n] *= w[:, None, None]


def zeros_first(torch, x):
    """(padding before the first token that counts, and behind the last one)"""
    for n, rows in (("v", slice(0, 70)), ("d_o", slice(60, 130))):
        x[n][rows] = 0
    x["state"][:] = x["d_state"][:] = 0


def small_first(torch, x):
    x["v"][:64] *= 2.0 ** -30
    x["d_o"][64:130] *= 2.0 ** -30
    x["state"] *= 2.0 ** -30
    x["d_state"] *= 2.0 ** -30


def large_first(torch, x):
    x["v"][64:130] *= 2.0 ** -8
    x["d_o"][:64] *= 2.0 ** -8
    x["state"] *= 2.0 ** -8
    x["d_state"] *= 2.0 ** -8


def one_large_value(torch, x):
    x["v"][100, 1, 5] = 2.0 ** 14
    x["d_o"][3, 2, 60] = 2.0 ** 14


@pytest.mark.parametrize("change", [zeros_first, small_first, large_first, one_large_value, gates_that_forget, gates_that_keep, betas_at_the_ends, betas_of_nothing, the_same_key, keys_in_turn, empty_keys, small, large, heads_of_all_sizes],
                         ids=lambda f: f.__name__)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
def test_values(gpu, change, dtype, d):
    # Rows 2^-30 of their sequence's largest are past fp16's smallest step, 2^-24 with the largest at 2^5: they come in off by up to 2^-25 / 2^5 times the largest (4 here) = 2^-28.
    # Products of these with rows of size one over d places: 2^-28 * sqrt(128) = 4.2e-8, times scale in dq and dk; dlog_f adds up 64 tokens.
    lost = {"dq": 4.2e-8, "dk": 4.2e-8, "dbeta": 4.2e-8, "dlog_f": 64 * 4.2e-8} if change is small_first and dtype == "bf16" else {}
    # d_state: scale gamma dO and gamma beta Y come in off by 2^-28 each (0.58 of it in deviation), times q's and k's 1/8 and the root of some 8 rows before gamma has fallen: 3.8e-9 at
    # five deviations from each, beside results that are 2^-8 of usual.
    if change is large_first and dtype == "bf16":
        lost = {"d_state": 7.6e-9, "state": 7.6e-9}      # (the last state: E and rho U, likewise)
    # Beside 2^14 at 2^5 a two-part operand is off by 2^-25 * 2^9 = 2^-16 whatever its size; three (S, E, U) come into a state over rows that gates of mean 0.88 weigh as some 10, times k's
    # largest 0.2: 9e-5.  (The token's own outcome is 2^14 large, but in one column and head.)
    if change is one_large_value and dtype == "bf16":
        # dk and dq add up products with that one column, Y S^T and dO S^T with S = 2^14 beta k = 1000 for values of size one, up to eight roundings of 2^-12 each and no averaging
        # over columns; dbeta = Y.E has the same factors (E of 2^14 * 0.2 by later keys' overlap), dlog_f three such.  dv has Y of the head with the large d_o, 2^14 * 0.125 scale.
        lost = {"state": 9e-5, "d_state": 9e-5, "dk": 8 * 2 ** -12 * 1000, "dq": 8 * 2 ** -12 * 1000 * d ** -0.5, "dbeta": 8 * 2 ** -12 * 3300, "dlog_f": 24 * 2 ** -12 * 3300, "dv": 8 * 2 ** -12 * 2000 * d ** -0.5,
                "o": 8 * 2 ** -12 * 1000 * d ** -0.5}

    def check(torch, name, got, want, cu, f32):
        for h in range(3):      # the first head has neither of the large values
            close(torch, name, got[:, h : h + 1], want[:, h : h + 1], cu, f32, least=lost.get(name, 1e-30) if h or change is not one_large_value else 1e-30)

    train(gpu, [130, 40], 3, 1, d, dtype, change=change, seed=8, check=check)


def pushes_one_way(torch, x):
    """Reflections (beta 2) about one key, values that alternate: every step adds 2 |v| to the state, and backwards to its gradient.  (v and d_o of one size, that their sums be known.)"""
    x["k"][:], x["q"][:] = x["k"][0], x["k"][0]
    x["beta"][:] = 2.0
    for n in ("v", "d_o"):
        x[n][:] = x[n][0].sign()
    x["state"][:] = x["d_state"][:] = 0
    x["v"][1::2] *= -1
    x["log_f"][:] = 0.0


@pytest.mark.parametrize("d", [64, 128])
def test_states_that_outgrow_their_operands(gpu, d):
    """A state 3000 times the values that come in: past what fp16 operands have room for at first.  bf16 keys are off unit length by up to 2^-8, so the reflections stretch by that: a longer run would
    grow without bound in any arithmetic."""
    torch, pa = gpu
    x = dm.batch([1500, 70], 2, 1, d, seed=1)
    pushes_one_way(torch, x)
    k = torch.zeros(d)
    k[: d // 4] = (d // 4) ** -0.5 if d == 64 else 0.17578125      # 16 of 1/4: of length one; 32 of 45/256: 0.9944
    x["k"][:], x["q"][:] = k.bfloat16(), k.bfloat16()
    y, scale = to_gpu(x), d ** -0.5
    o, last = pa.path_delta_fwd(y["q"], y["k"], y["v"], y["beta"], log_f=y["log_f"], scale=scale, cu_seqlens=y["cu"], max_len=1500, final_state=True)
    o1 = pa.path_delta_fwd(y["q"], y["k"], y["v"], y["beta"], log_f=y["log_f"], scale=scale, cu_seqlens=y["cu"], max_len=1500)
    want_o, want_last = dm.forward(x, scale)
    assert want_last.abs().max() > (700 if d == 64 else 10)
    close(torch, "o", o, want_o, [0, 1500, 1570], False)
    # The state adds up 64 alternating steps of 2 |E| a chunk, and the steps come of rows of P, sum_n 2 r^n in magnitude (r = 1 - 2 |k|^2), that cancel to one.  At d = 64 every number is a power of
    # two's multiple and exact.  At d = 128: r = -0.977, sum |P| = 66, |E| = 86, operands of two parts off by 2^-22 each: E off by up to 66 * 86 * 2 * 2^-22 = 2.7e-3, U = 2 E by 5.4e-3, the state
    # by 64 rows of 0.176 of it, times 1.28 for the chunks before: 0.078 if all fell one way, an eighth of it where 64 rows' are independent.
    if d == 64:
        close(torch, "state", last, want_last, [0, 1500, 1570], False)
    else:
        assert ((last.double().cpu() - want_last).abs() <= 0.078 / 8).all()
    # Without states, operands of 11 bits: E = v - S k is rounded to half a step of 2^-11 of itself, which is |v| where it is 1024 |v|, so from there on a step may be lost
    # whole (and all of a chunk's, whose roundings are alike).  That leaves o off by up to what the state grows behind that: |o| / (2 |v| t) for t steps, (1500 - 512) / 1500 of the largest.
    # At d = 128 (see above) 2^-12 takes the place of 2^-22, and o = scale q.S^T has 0.088 * 0.989 of 64 rows' error in U: 0.088 * 64 * 66 * 86 * 4 * 2^-12 * 1.28 / 8 = 5.0.
    off = (o1.double().cpu() - want_o).abs()
    if d == 64:
        assert off.max() <= 0.66 * want_o.abs().max() and off[:400].max() <= 2 * 8e-3 * want_o[:400].abs().max()
    else:
        assert off.max() <= 5.0


@pytest.mark.parametrize("back", [False, True])
def test_training_of_states_that_outgrow_their_operands(gpu, back):
    def change(torch, x):
        pushes_one_way(torch, x)
        if back:
            x["d_o"][1::2] *= -1
        k = torch.zeros(64)
        k[:16] = 0.25
        x["k"][:], x["q"][:] = k.bfloat16(), k.bfloat16()

    # A gradient is a chunk's first state's part and 64 rows of steps that alternate and are up to twice its size, through two operands of 11 bits: 64 * 2 * 2 * 2^-12 of the
    # largest result where all roundings fall one way, as those of equal rows do; dlog_f
    # adds up three of them, the state with its gradient among them, in which both factors grow: twice that.
    def check(torch, name, got, want, cu, f32):
        for a, b in zip(cu[:-1], cu[1:]) if "state" not in name else ((0, 1), (1, 2)):
            off = float((got.double().cpu() - want)[a:b].abs().max())
            assert off <= 2 ** (-3 if name == "dlog_f" else -4) * float(want[a:b].abs().max()) + 1e-30, (name, a, off, float(want[a:b].abs().max()))

    for n in (400, 1500):
        train(gpu, [n, 70], 2, 1, 64, change=change, without=False, check=check)


def test_rows_of_no_sequence(gpu):
    """Rows behind the last offset are left as they are, in o and in all gradients' tokens that the call does write whole tensors for."""
    torch, pa = gpu
    x = dm.batch([70, 9], 2, 2, 64, tail=50, seed=6)
    y, cu = to_gpu(x), x["cu"].tolist()
    o = torch.full_like(y["v"], 7.0)
    pa.path_delta_fwd(y["q"], y["k"], y["v"], y["beta"], log_f=y["log_f"], cu_seqlens=y["cu"], max_len=70, o=o)
    assert (o[cu[-1]:] == 7.0).all()
    close(torch, "o", o, dm.forward(x, 64 ** -0.5)[0], cu, False)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_bounds_hold(gpu, dtype):
    """Offsets past the tensors, offsets that fall, and sequences past max_len are held to them (nothing is read or written outside: the tensors end with the allocation)."""
    torch, pa = gpu
    x = dm.batch([100, 60], 2, 1, 64, dtype, seed=1)
    y = to_gpu(x)
    for cu, max_len, same in (([0, 100, 1000], 200, [0, 100, 160]), ([0, 100, 160], 90, None), ([-5, 100, 160], 160, [0, 100, 160]), ([0, 150, 20], 200, None)):
        c = torch.tensor(cu, dtype=torch.int32, device="cuda")
        o = torch.zeros_like(y["v"])
        pa.path_delta_fwd(y["q"], y["k"], y["v"], y["beta"], log_f=y["log_f"], cu_seqlens=c, max_len=max_len, o=o)
        torch.cuda.synchronize()
        if same is not None:
            close(torch, "o", o, dm.forward(x, 64 ** -0.5)[0], same, dtype == "fp32")
        elif max_len == 90:
            short = {**x, "cu": torch.tensor([0, 90])}
            close(torch, "o", o[:90], dm.forward(short, 64 ** -0.5)[0][:90], [0, 90], dtype == "fp32")
            assert (o[90:100] == 0).all()


def test_segments_are_the_whole(gpu):
    """A long sequence at once, and in segments through its states."""
    torch, pa = gpu
    x = dm.batch([700], 2, 2, 128, gate_mean=5.0, seed=3)
    y = to_gpu(x)
    at = lambda a, b: dict(cu_seqlens=torch.tensor([0, b - a], dtype=torch.int32, device="cuda"), max_len=b - a)
    call = lambda a, b, st: pa.path_delta_fwd(*[y[n][a:b].contiguous() for n in ("q", "k", "v", "beta")], log_f=y["log_f"][a:b].contiguous(), state_in=st, final_state=True, **at(a, b))
    o, last = call(0, 700, None)
    state, parts = None, []
    for a, b in ((0, 1), (1, 300), (300, 364), (364, 700)):
        p, state = call(a, b, state)
        parts.append(p)
    want_o, want_last = dm.forward(x, 128 ** -0.5)
    close(torch, "o", torch.cat(parts), want_o, [0, 700], False)
    close(torch, "o", o, want_o, [0, 700], False)
    close(torch, "state", state, want_last, [0, 700], False)
    # in place
    st = y["state"].clone()
    ref = pa.path_delta_fwd(*[y[n] for n in ("q", "k", "v", "beta")], log_f=y["log_f"], state_in=y["state"], final_state=True, cu_seqlens=y["cu"], max_len=700)
    got = pa.path_delta_fwd(*[y[n] for n in ("q", "k", "v", "beta")], log_f=y["log_f"], state_in=st, state_out=st, cu_seqlens=y["cu"], max_len=700)
    assert torch.equal(got[0], ref[0]) and torch.equal(st, ref[1])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lengths,H,G", [([2305], 1, 1), ([2400], 1, 3), ([5000], 1, 1), ([2700, 100, 0, 1600], 2, 1), ([769, 2304, 1, 768], 1, 1)], ids=str)
def test_cut_sequences(gpu, lengths, H, G, d, dtype):
    """Few heads and long sequences: cut into segments, with and without states; states carried on in place."""
    torch, pa = gpu
    x = dm.batch(lengths, H, G, d, dtype, seed=len(lengths) + H, gate_mean=6.0)
    y, scale, cu = to_gpu(x), d ** -0.5, x["cu"].tolist()
    for state in (None, "state"):
        st = x[state] if state else None
        want_o, want_last = dm.forward(x, scale, st)
        how = dict(log_f=y["log_f"], scale=scale, cu_seqlens=y["cu"], max_len=max(lengths))
        ins = [y[n] for n in ("q", "k", "v", "beta")]
        o = pa.path_delta_fwd(*ins, state_in=y[state] if state else None, workspace=poison(torch, pa, x, H, G, d, max(lengths), dtype, False), **how)
        close(torch, "o", o, want_o, cu, dtype == "fp32")
        own = y["state"].clone() if state else torch.full_like(y["state"], math.nan)
        o, last = pa.path_delta_fwd(*ins, state_in=own if state else None, state_out=own, workspace=poison(torch, pa, x, H, G, d, max(lengths), dtype, False), **how)
        close(torch, "o", o, want_o, cu, dtype == "fp32")
        close(torch, "state", last, want_last, cu, dtype == "fp32")
        again = pa.path_delta_fwd(*ins, state_in=y[state] if state else None, final_state=True, **how)
        assert torch.equal(again[0], o) and torch.equal(again[1], last)


def test_infinities_and_nan_stay_in_their_head_and_sequence(gpu):
    """What is not finite shows in no other sequence or head, and, by chunks, in no chunk before its own."""
    torch, pa = gpu
    for n in ("q", "k", "v", "beta", "log_f"):
        for bad in (math.inf, math.nan):
            x = dm.batch([200, 100], 3, 1, 64, seed=2)
            y = to_gpu(x)
            how = dict(cu_seqlens=y["cu"], max_len=200, final_state=True)
            call = lambda: pa.path_delta_fwd(y["q"], y["k"], y["v"], y["beta"], log_f=y["log_f"], **how)
            o, last = call()
            y[n][140, 1] = bad
            o1, last1 = call()
            keep = torch.ones(300, 3, dtype=torch.bool, device="cuda")
            keep[128:200, 1] = False
            assert torch.equal(o1[keep], o[keep]), (n, bad)
            assert torch.equal(last1[1], last[1]) and torch.equal(last1[0, [0, 2]], last[0, [0, 2]])


def test_bits_streams_and_threads(gpu):
    """The same bits on another stream, with memory of that stream, and from two threads at once."""
    import threading
    torch, pa = gpu
    x = dm.batch([300, 77, 130], 4, 2, 128, seed=5)
    y = to_gpu(x)
    need = pa.path_delta_workspace_bytes(3, 507, 300, 4, 2, 128, 1, True)

    def step(stream=None):
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        how = dict(log_f=y["log_f"], cu_seqlens=y["cu"], max_len=300, workspace=ws, state_in=y["state"], stream=stream)
        out = pa.path_delta_train_fwd(y["q"], y["k"], y["v"], y["beta"], final_state=True, **how)
        return (*out, *pa.path_delta_train_bwd(y["q"], y["k"], y["v"], y["beta"], y["d_o"], d_state_out=y["d_state"], **how))

    want = step()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = step(s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    results = {}

    def work(i):
        st = torch.cuda.Stream()
        with torch.cuda.stream(st):
            results[i] = [step() for _ in range(5)]
        st.synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(3)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert len(results) == 3
    for r in results.values():
        assert all(torch.equal(a, b) for got in r for a, b in zip(got, want))


def test_captured(gpu):
    """A training step captured into a graph, replayed with other inputs and other lengths; the program's own work between the replays."""
    torch, pa = gpu
    x = dm.batch([150, 64, 30], 2, 2, 64, seed=1, tail=20)
    y = to_gpu(x)
    ws = torch.empty(pa.path_delta_workspace_bytes(3, 264, 264, 2, 2, 64, 1, True), dtype=torch.uint8, device="cuda")

    def step(ws):
        how = dict(log_f=y["log_f"], cu_seqlens=y["cu"], max_len=264, workspace=ws, state_in=y["state"])
        out = pa.path_delta_train_fwd(y["q"], y["k"], y["v"], y["beta"], final_state=True, **how)
        return (*out, *pa.path_delta_train_bwd(y["q"], y["k"], y["v"], y["beta"], y["d_o"], d_state_out=y["d_state"], **how))

    step(ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(ws)
    for i, cu in enumerate(([0, 150, 214, 244], [0, 10, 100, 264], [0, 0, 264, 264], [0, 150, 214, 244])):
        z = to_gpu(dm.batch([150, 64, 30], 2, 2, 64, seed=10 + i, tail=20))
        for n in ("q", "k", "v", "beta", "log_f", "d_o", "state", "d_state"):
            y[n].copy_(z[n])
        y["cu"].copy_(torch.tensor(cu, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        want = step(torch.full_like(ws, 255))
        for a, b in zip(got, want):
            rows = slice(0, cu[-1]) if a.shape[0] == 264 else slice(None)
            assert torch.equal(a[rows], b[rows])


def test_two_graphs_with_one_workspace(gpu):
    """Two captured steps share a workspace, replayed in turn on one stream."""
    torch, pa = gpu
    data = [to_gpu(dm.batch([100, 30], 2, 1, 64, seed=s)) for s in (1, 2)]
    ws = torch.empty(pa.path_delta_workspace_bytes(2, 130, 100, 2, 1, 64, 1, True), dtype=torch.uint8, device="cuda")

    def step(y, ws):
        how = dict(log_f=y["log_f"], cu_seqlens=y["cu"], max_len=100, workspace=ws)
        return (pa.path_delta_train_fwd(y["q"], y["k"], y["v"], y["beta"], **how), *pa.path_delta_train_bwd(y["q"], y["k"], y["v"], y["beta"], y["d_o"], **how))

    want = [step(y, torch.empty_like(ws)) for y in data]
    graphs = []
    for y in data:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step(y, ws)
        graphs.append((g, out))
    for _ in range(3):
        for (g, out), w in zip(graphs, want):
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, w))


@pytest.mark.parametrize("layout", [0, 1])
def test_far_rows(gpu, layout):
    """Values of more than 2^31 elements: the last heads and tokens against a call on them alone."""
    torch, pa = gpu
    L, V, d = 131100, 130, 128
    g = torch.Generator(device="cuda").manual_seed(1)
    unit = lambda *s: torch.nn.functional.normalize(torch.randn(*s, device="cuda", generator=g), dim=-1).bfloat16()
    heads = lambda n, *m: (1, n, L, *m) if layout == 0 else (1, L, n, *m)
    q, k = unit(*heads(1, d)), unit(*heads(1, d))
    v = torch.randn(*heads(V, d), device="cuda", generator=g, dtype=torch.bfloat16)
    assert v.numel() > 1 << 31
    beta = torch.rand(*heads(V), device="cuda", generator=g).bfloat16()
    o, last = pa.path_delta_fwd(q, k, v, beta, layout=layout, final_state=True)
    pick = (lambda t: t[:, -1:].contiguous()) if layout == 0 else (lambda t: t[:, :, -1:].contiguous())
    o1, last1 = pa.path_delta_fwd(q, k, pick(v), pick(beta), layout=layout, final_state=True)
    # (one head alone is cut into segments: two results, each off by the bars above)
    a, b = pick(o).flatten(0, 2).float(), o1.flatten(0, 2).float()
    assert b.std() > 0.01 and ((a - b).abs() <= 2 * (E16 * b.abs() + 8e-3 * b.square().mean().sqrt())).all()
    assert ((last[:, -1:] - last1).abs() <= 2e-5 * last1.square().mean().sqrt()).all()
