"""Weight sums and eviction on the GPU against the definitions (sums in 64 bits, eviction to the bit)."""
import math

import pytest
import torch

from paper_2401_06706_amd import binding as M
from tests import chunk_ref as R
from tests.test_gpu_chunk import DEV, SHAPES, gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("last", [0, 1, 33])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_weight_sums(shape, dtype, last):
    lens, news, H_q, H_kv, d, page = shape
    batch = R.make_batch(gen(1), DEV, dtype, lens, news, H_q, H_kv, d, page)
    scale = 1 / math.sqrt(d)
    _, _, lse, _ = R.attention(batch, scale, dtype)
    lse = lse.float()
    sums = torch.rand(len(lens), H_kv, batch["capacity"], generator=gen(2)).to(DEV)
    for b, (L, n) in enumerate(zip(lens, news)):
        sums[b, :, L:L + n] = float("nan")                # nothing of what stands at the places of new tokens counts
        sums[b, :, L + n:] = 3.0
    before = sums.clone()
    want, bound = R.weight_sums(batch, scale, lse, sums, last)
    M.mcsd_attn_weight_sums(M.weight_sums_args(batch["q"], batch["k_pool"], batch["table"], batch["chunk_start"], batch["prefix_len"], lse, sums,
                                               scale, last))
    torch.cuda.synchronize()
    for b, (L, n) in enumerate(zip(lens, news)):
        if n == 0:
            assert torch.equal(sums[b], before[b])
            continue
        assert (sums[b, :, L + n:] == 3.0).all()
        err = (sums[b, :, :L + n].double() - want[b, :, :L + n]).abs()
        assert (err <= bound[b, :, :L + n]).all(), f"{float(err.max())} {torch.nonzero(~(err <= bound[b, :, :L + n]))[:4].tolist()}"


def evict_case(lens, keeps, first, recent, layers, H_kv, d, dtype, page, fresh, values, seed=1, capacity=None):
    g = gen(seed)
    B = len(lens)
    cap = capacity or max(1, -(-max(lens) // page)) * page
    width = -(-cap // page)
    n_pages = 2 * B * width + 1
    order = torch.randperm(n_pages, generator=g)[:2 * B * width].int()
    table, other = order[:B * width].view(B, width), order[B * width:].view(B, width)
    lead = () if layers is None else (layers,)
    k = torch.randn(*lead, n_pages, H_kv, page, d, generator=g).to(dtype)
    v = torch.randn(*lead, n_pages, H_kv, page, d, generator=g).to(dtype)
    sums = values(torch.rand(*lead, B, H_kv, cap, generator=g))
    kept = torch.full(sums.shape, -7, dtype=torch.int32)
    want_k, want_v, want_s, want_kept = k.clone(), v.clone(), sums.clone(), kept.clone()
    to = other if fresh else table
    for l in range(layers or 1):
        at = (lambda t: t) if layers is None else (lambda t: t[l])
        for b, n in enumerate(lens):
            for h in range(H_kv):
                pos = R.evicted(n, keeps[b], first, recent, at(sums)[b, h].tolist())
                for j, i in enumerate(pos):
                    sp, sr, dp, dr = int(table[b, i // page]), i % page, int(to[b, j // page]), j % page
                    at(want_k)[dp, h, dr] = at(k)[sp, h, sr]
                    at(want_v)[dp, h, dr] = at(v)[sp, h, sr]
                    at(want_s)[b, h, j] = at(sums)[b, h, i]
                    at(want_kept)[b, h, j] = i
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    k, v, sums, kept, flags = k.to(DEV), v.to(DEV), sums.to(DEV), kept.to(DEV), i32([77] * B)
    prefix = i32(lens)
    M.mcsd_kv_evict_paged(M.evict_args(k, v, table.to(DEV), sums, prefix, i32(keeps), kept, flags, first, recent, other.to(DEV) if fresh else None))
    torch.cuda.synchronize()
    assert prefix.tolist() == [min(n, max(0, c)) for n, c in zip(lens, keeps)] and flags.tolist() == [0] * B
    assert torch.equal(kept.cpu(), want_kept)
    bits = lambda t: t.cpu().contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)
    for got, want in [(k, want_k), (v, want_v), (sums, want_s)]:
        assert torch.equal(bits(got), bits(want))


def some_zero(x):
    return torch.where(x < 0.5, torch.zeros_like(x), torch.round(x * 16) / 16)


def any_number(x):
    y = x.clone().flatten()
    y[::7], y[1::11], y[2::13], y[3::17] = float("nan"), float("inf"), -float("inf"), -0.0
    return y.view(x.shape) - 0.25


CASES = [  # lens, keeps, first, recent, layers, H_kv, d, page
    ([1], [1], 0, 0, None, 1, 8, 32),
    ([5], [0], 2, 2, None, 2, 64, 32),
    ([100, 40, 0, 64], [40, 41, 3, 64], 4, 8, None, 2, 64, 32),
    ([300, 299], [128, 1], 0, 0, 2, 3, 96, 96),
    ([300], [100], 60, 60, 2, 1, 128, 64),
    ([1500, 700], [600, 650], 4, 128, 2, 2, 128, 64),
    ([65, 64, 63], [64, 1, -5], 0, 1, 1, 2, 80, 32),
    ([2100], [2099], 0, 0, None, 1, 256, 32),
]


@pytest.mark.parametrize("values", [lambda x: x, some_zero, any_number, torch.zeros_like, lambda x: -x])
@pytest.mark.parametrize("fresh", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_evict(case, fresh, values):
    lens, keeps, first, recent, layers, H_kv, d, page = case
    evict_case(lens, keeps, first, recent, layers, H_kv, d, torch.bfloat16, page, fresh, values)


@pytest.mark.parametrize("fresh", [False, True])
def test_evict_fp32(fresh):
    evict_case([700, 33], [257, 32], 1, 5, 2, 2, 36, torch.float32, 32, fresh, some_zero)


@pytest.mark.parametrize("fresh", [False, True])
def test_evict_long(fresh):
    """More positions than the registers of a workgroup hold."""
    evict_case([40001, 16385], [9000, 16384], 4, 100, None, 1, 8, torch.bfloat16, 256, fresh, some_zero, capacity=40192)


def test_evict_bad_pages():
    """Rows in or for pages outside the pool are not moved and flag their sequence; the others are served."""
    page, d, B = 32, 64, 2
    k = torch.randn(9, 1, page, d, generator=gen(1)).to(torch.bfloat16).to(DEV)
    v = k + 1
    table = torch.tensor([[0, -1, 2, 3], [4, 5, 6, 7]], dtype=torch.int32, device=DEV)
    sums = torch.arange(128.0, device=DEV).repeat(B, 1, 1)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    kept, flags, prefix, k0 = torch.zeros(B, 1, 128, dtype=torch.int32, device=DEV), i32([0, 0]), i32([128, 128]), k.clone()
    M.mcsd_kv_evict_paged(M.evict_args(k, v, table, sums, prefix, i32([64, 64]), kept, flags, 0, 0))
    torch.cuda.synchronize()
    assert flags.tolist() == [M.FLAG_BAD_PAGES, 0] and prefix.tolist() == [64, 64]
    assert torch.equal(k[0], k0[2]) and torch.equal(k[4], k0[6]) and torch.equal(k[5], k0[7]) and torch.equal(k[8], k0[8])
    assert kept[0, 0, :64].tolist() == list(range(64, 128))
