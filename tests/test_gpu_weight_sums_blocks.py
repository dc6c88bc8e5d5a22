"""Weight sums where a workgroup takes two or four blocks of 128 positions (few rows a sequence, many workgroups): one tile of rows and several, new
positions on both sides of a workgroup's border, more rows than are summed up at once."""
import math

import pytest
import torch

from paper_2401_06706_amd import binding as M
from tests import chunk_ref as R
from tests.test_gpu_chunk import DEV, gen

pytestmark = pytest.mark.gpu

SHAPES = [  # lens, news, H_q, H_kv, d
    ([0, 127, 128, 511, 512, 513, 1100, 3], [1] * 8, 8, 2, 128),
    ([700, 0, 255, 256, 20, 900, 130, 480], [1, 1, 1, 1, 1, 0, 1, 60], 8, 2, 128),      # eight tiles of rows in one sequence, 540 keys
    ([500, 250, 1000, 380], [30, 20, 25, 10], 4, 2, 64),
    ([100, 600, 254], [9, 16, 2], 6, 2, 80),
    ([300, 1030], [1, 40], 3, 3, 256),
    ([130] * 39 + [520], [1] * 39 + [600], 4, 1, 32),                                   # 2400 rows: more than 64 tiles
]


@pytest.mark.parametrize("last", [0, 1, 7])
@pytest.mark.parametrize("groups", [4096, 8192])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_blocks(shape, dtype, groups, last):
    lens, news, H_q, H_kv, d = shape
    B = len(lens)
    assert sum(news) * H_q // H_kv <= 64 * B
    batch = R.make_batch(gen(71), DEV, dtype, lens, news, H_q, H_kv, d, 32)
    table = torch.full((B, -(-groups * 128 // (B * H_kv) // 32) + 1), -1, dtype=torch.int32, device=DEV)
    table[:, :batch["table"].shape[1]] = batch["table"]
    batch["table"], batch["capacity"] = table, table.shape[1] * 32
    assert groups <= B * H_kv * -(-batch["capacity"] // 128) < 2 * groups
    scale = 1 / math.sqrt(d)
    lse = R.attention(batch, scale, dtype)[2].float()
    sums = torch.rand(B, H_kv, batch["capacity"], generator=gen(72)).to(DEV)
    for b, (L, n) in enumerate(zip(lens, news)):
        sums[b, :, L:L + n] = float("nan")                # nothing of what stands at the places of new tokens counts
        sums[b, :, L + n:] = 3.0
    before = sums.clone()
    want, bound = R.weight_sums(batch, scale, lse, sums, last)
    M.mcsd_attn_weight_sums(M.weight_sums_args(batch["q"], batch["k_pool"], batch["table"], batch["chunk_start"], batch["prefix_len"], lse, sums, scale, last))
    torch.cuda.synchronize()
    for b, (L, n) in enumerate(zip(lens, news)):
        if n == 0:
            assert torch.equal(sums[b], before[b])
            continue
        assert (sums[b, :, L + n:] == 3.0).all()
        err = (sums[b, :, :L + n].double() - want[b, :, :L + n]).abs()
        assert (err <= bound[b, :, :L + n]).all(), f"{b} {float(err.max())} {torch.nonzero(~(err <= bound[b, :, :L + n]))[:4].tolist()}"
