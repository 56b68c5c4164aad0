"""The wide model agrees with paged_model.py, and the bars of paged_wide.py tell operands kept as two bf16 numbers from operands kept as one (the mistake is planted in
the model; no GPU)."""
import pytest
import torch

import paged_model as pm
import paged_wide as wide

CASES = [
    # old, new, H, G, d
    ([300, 129, 15], [1, 5, 16], 2, 1, 128),
    ([300, 129], [8, 3], 2, 4, 64),
    ([129, 70], [65, 63], 1, 2, 128),
    ([1100], [257], 1, 1, 64),
    ([500, 50], [130, 1], 2, 1, 128),
]


def one(u):
    return u.float().bfloat16().double()


def two(u):
    hi = u.float().bfloat16()
    return hi.double() + (u.float() - hi.float()).bfloat16().double()


@pytest.mark.parametrize("gates", [False, True])
@pytest.mark.parametrize("op", ["attn", "append", "extend"])
def test_models_agree(op, gates):
    x = wide.batch([40, 0, 7], [5, 30, 0], 2, 3, 64, 16, "bf16", gates, seed=1, device="cpu")
    a, b = wide.expect(x, 0.125, op), pm.expect(x, 0.125, op)
    if op != "append":
        assert (a[0] - b[0]).abs().max() < 1e-12 and (a[1] - b[1]).abs().max() < 1e-12
    for p, q in zip(a[3:], b[2:]):
        if p is not None:
            assert torch.equal(p.isnan(), q.isnan()) and (p.double() - q.double()).nan_to_num().abs().max() < 1e-5


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-{c[1]}-{c[4]}".replace(" ", ""))
def test_a_lost_part_of_x_exceeds_the_bar_of_lse(case):
    old, new, H, G, d = case
    x = wide.batch(old, new, H, G, d, 32, "bf16", seed=sum(old), device="cpu")
    lse = wide.expect(x, d ** -0.5, "attn")[1]
    bar = wide.bars(x)[1]
    off = lambda change: float((wide.expect(x, d ** -0.5, "attn", change)[1] - lse).abs().max())
    assert off(two) < bar / 2
    assert off(one) > 2 * bar


@pytest.mark.parametrize("case", CASES[2:], ids=lambda c: f"{c[0]}-{c[1]}-{c[4]}".replace(" ", ""))
def test_a_lost_part_of_the_transitions_exceeds_the_bar_of_keys(case):
    """New keys carried through the tiles as one bf16 number a tile, and as two; cached keys with a matrix of one bf16 number."""
    old, new, H, G, d = case
    x = wide.batch(old, new, H, G, d, 32, "bf16", seed=sum(old), device="cpu")
    _, _, bar, chunk = wide.bars(x)
    assert chunk
    cu = x["cu_new"].tolist()
    worst = {one: 0.0, two: 0.0}
    matrix = 0.0
    for s, n in enumerate(old):
        t0, m = cu[s], cu[s + 1] - cu[s]
        k, w, b = (x[i][t0:t0 + m].double().transpose(0, 1) for i in ("k", "w", "beta"))
        step = lambda y, t: y - b[:, t, None, None] * (y * w[:, t, None]).sum(-1, keepdim=True) * w[:, t, None]

        def carried(change):
            y = k.clone()
            for t in range(m):
                y[:, :t] = step(y[:, :t], t)
                if t % 64 == 63:
                    y[:, :t + 1] = change(y[:, :t + 1])
            return y
        exact = carried(lambda y: y)
        for change in worst:
            worst[change] = max(worst[change], float(((carried(change) - exact).abs() - 2 ** -8 * exact.abs()).max()))
        if m > 16:
            M = torch.eye(d, dtype=torch.float64).repeat(H, 1, 1)      # rows e_i carried on: the transpose of what keys meet
            for t in range(m):
                M = step(M, t)
            M -= torch.eye(d, dtype=torch.float64)
            K, = wide.cached(x, s, ("kpages",))
            y = K + K @ M
            matrix = max(matrix, float(((K @ (one(M) - M)).abs() - 2 ** -8 * y.abs()).max()))
    assert worst[two] < bar / 2
    assert worst[one] > 2 * bar
    assert matrix > bar + wide.HALF
