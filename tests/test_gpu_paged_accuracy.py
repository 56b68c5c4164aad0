"""The paged calls on the GPU to the documented accuracy (bars: paged_wide.py), at small sizes and at those that reach every form of the kernels: 32 and 64 rows of a
tile in one workgroup of the sweep, with and without the append's scan, pieces of one step up to those whose page numbers are fetched more than once."""
import pytest

import paged_wide as wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    import paper_2505_16381_amd as pa
    assert torch.cuda.is_available()
    pa.load_library()
    return torch, pa


def check(gpu, op, old, new, H, G, d, page, dtype, gates, seed):
    torch, pa = gpu
    x = wide.batch(old, new, H, G, d, page, dtype, gates, seed)
    y = {n: t.clone() if t is not None else None for n, t in x.items()}
    kvwb = (y["k"], y["v"], y["w"], y["beta"])
    cache = (y["kpages"], y["vpages"], y["page_table"], y["cached"], y["cu_new"], max(new), max(old))
    more = dict(log_f=y["log_f"], cpages=y["cpages"])
    scale = d ** -0.5
    got = None
    if op == "append":
        pa.path_paged_append(*kvwb, *cache, **more)
    else:
        got = (pa.path_paged_attn if op == "attn" else pa.path_paged_extend)(y["q"], *kvwb, *cache, scale=scale, **more)
    torch.cuda.synchronize()
    print(op, old, new, flush=True)
    wide.compare(x, y, got, wide.expect(x, scale, op), op)
    torch.cuda.empty_cache()


ids = lambda c: f"{str(c[0])[:20]}-{str(c[1])[:20]}-{c[2]}x{c[3]}".replace(" ", "")

SMALL = [
    # old, new, H, G, page
    ([0], [1], 1, 1, 16),
    ([300, 129, 15], [1, 5, 16], 2, 1, 32),
    ([300, 129], [8, 3], 2, 4, 16),
    ([3000, 33], [2, 1], 1, 2, 64),
    ([129, 70], [65, 63], 1, 2, 32),
    ([1100], [257], 1, 1, 128),
    ([500, 50, 700], [130, 1, 5], 2, 1, 64),
    ([0], [200], 2, 3, 16),
]


@pytest.mark.parametrize("op", ["attn", "append", "extend"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", SMALL, ids=ids)
def test_documented_accuracy(gpu, case, d, dtype, op):
    old, new, H, G, page = case
    check(gpu, op, old, new, H, G, d, page, dtype, len(old) == 3, seed=sum(old) + d)


# The sweep: (T / 64 + 1) * H * G up to 272 takes 32 rows a workgroup, above 64; the append alone by nseq * H * d, up to 8192 and above.
SWEEP = [
    # old, new, H, G, page
    ([100], [1000], 16, 1, 64),         # 256: 32 rows, sixteen tiles
    ([100], [300], 64, 1, 64),          # 320: 64 rows; append 4096 (d = 64), 8192
    ([70, 0, 33], [200, 90, 20], 64, 1, 32),      # 64 rows; append 12288, 24576
    ([90, 40], [150, 3], 16, 8, 128),             # 64 rows, groups
    ([0], [1500], 16, 1, 64),           # 64 rows, 24 tiles
]


@pytest.mark.parametrize("op", ["attn", "append", "extend"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", SWEEP, ids=ids)
def test_both_row_counts_of_the_sweep(gpu, case, d, op):
    old, new, H, G, page = case
    check(gpu, op, old, new, H, G, d, page, "bf16", len(old) == 3, seed=sum(new) + d)


def test_sweep_of_many_tiles(gpu):
    check(gpu, "extend", [500], [2048], 16, 1, 64, 128, "bf16", True, seed=3)


@pytest.mark.parametrize("op", ["attn", "append", "extend"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", [([900] * 3, [70, 1, 33], 4, 2, 64), ([0], [700], 8, 1, 64)], ids=ids)
def test_fp32_and_bf16_chunks_of_several_heads(gpu, case, dtype, op):
    old, new, H, G, page = case
    check(gpu, op, old, new, H, G, 128, page, dtype, True, seed=4)


# Few new tokens with the whole cache in one piece: as many heads as fill the chip.  128 tokens a step of four waves (fp32, and both operations at d = 128: 64).
WALKS = [
    # old, new, H, G, d, page, dtype, gates
    ([1100, 700, 900, 31, 1000, 128, 129, 1090], [1] * 8, 64, 1, 64, 64, "bf16", True),
    ([700, 650, 500, 3, 513, 128, 129, 690], [1, 2, 4, 1, 16, 1, 1, 3], 64, 1, 128, 32, "bf16", False),
    ([700, 650, 500, 3], [3, 1, 8, 2], 64, 4, 128, 32, "bf16", True),             # up to 32 rows
    ([700, 650, 500, 3], [13, 1, 8, 2], 64, 4, 64, 16, "bf16", False),            # up to 64
    ([700, 650, 500, 3], [2, 1, 5, 3], 128, 1, 64, 32, "fp32", True),
    ([9000] + [40] * 7, [1] * 8, 64, 1, 64, 256, "bf16", False),                  # page numbers fetched twice (64 steps)
    ([5000] + [40] * 7, [2] * 8, 64, 1, 128, 256, "bf16", True),
    ([4700] + [40] * 3, [3] * 4, 64, 4, 64, 128, "fp32", False),
    ([8400] + [40] * 15, [2] * 16, 128, 1, 64, 256, "bf16", False),               # the append alone: one piece from 2048 heads on
]


@pytest.mark.parametrize("op", ["attn", "append", "extend"])
@pytest.mark.parametrize("case", WALKS, ids=lambda c: ids(c) + f"-{c[4]}-{c[6]}")
def test_long_walks_of_few_tokens(gpu, case, op):
    old, new, H, G, d, page, dtype, gates = case
    check(gpu, op, old, new, H, G, d, page, dtype, gates, seed=sum(new) + d)


# A chunk's cached part: pieces of more than 64 stages (4096 tokens) of the attention, keys carried on by workgroups of 128 up to 4096 tokens.
PIECES = [
    # old, new, H, G, d, dtype, gates
    ([4500], [130], 64, 8, 64, "bf16", False),
    ([4500], [130], 64, 8, 128, "bf16", True),
    ([2100], [130], 16, 2, 128, "bf16", False),
    ([5000, 4097, 100, 0], [17, 20, 18, 17], 64, 1, 128, "bf16", False),       # 4096 tokens a workgroup, a second one behind it
    ([5000, 4097, 100, 0], [17, 20, 18, 17], 64, 1, 64, "bf16", True),
    ([4500], [130], 64, 8, 64, "fp32", True),
    ([5000, 4097], [17, 20], 128, 1, 64, "fp32", False),
]


@pytest.mark.parametrize("op", ["attn", "append", "extend"])
@pytest.mark.parametrize("case", PIECES, ids=lambda c: ids(c) + f"-{c[4]}-{c[5]}")
def test_long_pieces_of_a_chunks_cache(gpu, case, op):
    old, new, H, G, d, dtype, gates = case
    check(gpu, op, old, new, H, G, d, 128, dtype, gates, seed=sum(new) + d)
