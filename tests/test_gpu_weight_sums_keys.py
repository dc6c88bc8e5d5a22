"""Weight sums where a key holds an infinity: a position that every row scores at -infinity is given nothing by them, however many
rows there are."""
import math

import pytest
import torch

from paper_2401_06706_amd import binding as M
from tests import chunk_ref as R
from tests.test_gpu_chunk import DEV, check, gen

pytestmark = pytest.mark.gpu

SHAPES = [  # lens, news, H_q, H_kv, d: rows per KV head 4, 32, 36, 1, 33 and 70 among them, a multiple of 32 or not
    ([50, 7], [1, 8], 8, 2, 128),
    ([50, 300, 40], [9, 1, 33], 4, 1, 128),
    ([90, 64], [70, 32], 2, 2, 64),
    ([40], [10], 10, 2, 80),
    ([45, 200], [1, 5], 3, 1, 256),
]


@pytest.mark.parametrize("last", [0, 1, 3])
@pytest.mark.parametrize("long", [False, True])         # (a capacity with which a workgroup takes several blocks of keys)
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_infinite_keys(shape, long, dtype, last):
    lens, news, H_q, H_kv, d = shape
    batch = R.make_batch(gen(41), DEV, dtype, lens, news, H_q, H_kv, d, 32)
    batch["q"][..., 3] = batch["q"][..., 3].abs() + 0.5
    at = [(b, j) for b, L in enumerate(lens) for j in (1, L - 1, L)]
    for b, j in at:
        batch["k_pool"][int(batch["table"][b, j // 32]), :, j % 32, 3] = -math.inf
    if long:
        table = torch.full((len(lens), 2 ** 20 // (len(lens) * H_kv) // 32 + 1), -1, dtype=torch.int32, device=DEV)
        table[:, :batch["table"].shape[1]] = batch["table"]
        batch["table"], batch["capacity"] = table, table.shape[1] * 32
        assert len(lens) * H_kv * -(-batch["capacity"] // 128) >= 8192 and sum(news) * H_q // H_kv <= 64 * len(lens)
    scale = 1 / math.sqrt(d)
    _, _, lse, _ = R.attention(batch, scale, dtype)
    lse = lse.float()
    assert torch.isfinite(lse).all()
    sums = torch.rand(len(lens), H_kv, batch["capacity"], generator=gen(42)).to(DEV)
    want, bound = R.weight_sums(batch, scale, lse, sums, last)
    for b, j in at:                                     # exp(-infinity), added to what was there
        want[b, :, j], bound[b, :, j] = 0.0 if j >= lens[b] else sums[b, :, j].double(), 0.0
    assert torch.isfinite(want).all() and torch.isfinite(bound).all()
    M.mcsd_attn_weight_sums(M.weight_sums_args(batch["q"], batch["k_pool"], batch["table"], batch["chunk_start"], batch["prefix_len"], lse, sums,
                                               scale, last))
    torch.cuda.synchronize()
    err = (sums.double() - want).abs()
    assert (err <= bound).all(), f"{torch.nonzero(~(err <= bound))[:4].tolist()}"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_of_infinite_keys(dtype, monkeypatch):
    """The attention before it agrees: such a key has no weight, and its value does not count."""
    batch = R.make_batch(gen(43), DEV, dtype, [50, 7], [9, 33], 4, 2, 128, 32)
    batch["q"][..., 3] = batch["q"][..., 3].abs() + 0.5
    for b, j in ((0, 1), (0, 49), (1, 30)):
        batch["k_pool"][int(batch["table"][b, j // 32]), :, j % 32, 3] = -math.inf
    plain = R.scores
    # (its score is exact: the errors are those of the other keys)
    monkeypatch.setattr(R, "scores", lambda *a: ((s, seen, torch.where(torch.isinf(mag), torch.zeros_like(mag), mag)) for s, seen, mag in plain(*a)))
    check(batch, 0.1, dtype)
