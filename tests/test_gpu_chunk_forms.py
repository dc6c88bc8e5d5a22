"""The forms that chunk attention, weight sums and eviction take by sizes and lengths: 32, 128 and 256 rows a workgroup, mixed batches in
one kernel or two, more sequences than a wavefront has lanes, more pages than it has, pools beyond 32-bit offsets, other orders of rows."""
import math

import pytest
import torch

from paper_2401_06706_amd import binding as M
from tests import chunk_ref as R
from tests.test_gpu_chunk import DEV, check, gen, run
from tests.test_gpu_evict import evict_case, some_zero

pytestmark = pytest.mark.gpu


def batch(seed, dtype, lens, news, H_q, H_kv, d, page):
    return R.make_batch(gen(seed), DEV, dtype, lens, news, H_q, H_kv, d, page)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [36, 64, 80, 96, 112, 128, 200, 256])
@pytest.mark.parametrize("news", [[1] * 12, [1] * 11 + [60], [20] * 12, [0, 3] * 6])
def test_rows_of_a_workgroup(news, d, dtype):
    """32 rows (few on average; one sequence with several tiles of them) and 128, keys in one piece and cut."""
    if dtype == torch.bfloat16 and d % 8:
        d += 4
    lens = [0, 5, 31, 32, 33, 700, 64, 1, 95, 300, 257, 1000]
    check(batch(21, dtype, lens, news, 6, 2, d, 32), 1 / math.sqrt(d), dtype)


@pytest.mark.parametrize("lens,news", [
    ([3000] * 5 + [0], [1] * 5 + [200]),        # the decoding sequences have most of the work: all in the kernel for few rows
    ([3000] * 5 + [4000], [1] * 5 + [200]),     # the other one has
    ([100, 0, 90, 3], [60, 1, 40, 64]),
    ([5, 2500], [250, 6]),
])
def test_mixed(lens, news):
    check(batch(22, torch.bfloat16, lens, news, 8, 2, 128, 64), 0.09, torch.bfloat16)


@pytest.mark.parametrize("B,long", [(70, 40), (70, 130), (140, 70)])
def test_many_sequences_of_many_rows(B, long):
    lens = [(53 * b) % 400 for b in range(B)]
    news = [0 if b % 6 == 5 else 1 if b % 3 == 1 else long for b in range(B)]
    check(batch(23, torch.bfloat16, lens, news, 8, 2, 128, 32), 0.09, torch.bfloat16)


def test_more_pages_than_lanes():
    """A workgroup of many rows walks through more pages than it holds entries of at once."""
    check(batch(24, torch.bfloat16, [8000, 7000], [600, 600], 4, 4, 128, 32), 0.09, torch.bfloat16)


@pytest.mark.parametrize("H_kv,news", [(2, [300]), (1, [40, 1]), (64, [70, 80, 90])])
def test_no_number_behind_a_long_prefix(H_kv, news):
    """Keys cut or not: what is no number reaches the rows that see it, and only those."""
    lens = [3000, 200, 0][:len(news)]
    b = batch(25, torch.bfloat16, lens, news, 2 * H_kv, H_kv, 128, 32)
    clean, clean_lse = run(b, 0.1)
    clean, clean_lse = clean.clone(), clean_lse.clone()
    for pos in (10, lens[0] - 1, lens[0], lens[0] + news[0] // 2, lens[0] + news[0] - 1):
        page, row = int(b["table"][0, pos // 32]), pos % 32
        old = b["v_pool"][page, 0, row].clone()
        b["v_pool"][page, 0, row, 17], b["v_pool"][page, 0, row, 90] = float("inf"), float("nan")
        out, lse = run(b, 0.1)
        first = max(0, pos - lens[0])
        want = clean.clone()
        want[first:news[0], :2, 17], want[first:news[0], :2, 90] = float("inf"), float("nan")
        assert torch.equal(lse, clean_lse) and torch.equal(torch.nan_to_num(out.float(), nan=-1e30), torch.nan_to_num(want.float(), nan=-1e30))
        b["v_pool"][page, 0, row] = old


@pytest.mark.parametrize("news", [[1, 1, 1], [100, 1, 260]])
def test_orders_of_rows(news):
    """q as a slice of a wider row and as rows of its own; nothing of what stands behind the last token is read or written."""
    b = batch(26, torch.bfloat16, [70, 5, 900], news, 8, 2, 128, 32)
    T = sum(news)
    packed, lse = run(dict(b, q=b["q"].contiguous()), 0.1)
    packed = packed.clone()
    wide = torch.full((T + 40, 3, 8, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:T, 1] = b["q"]
    out, lse2 = run(dict(b, q=wide[:, 1]), 0.1)         # (a padded batch: T is more than the sequences hold)
    _, bound, _, lse_bound = R.attention(b, 0.1, torch.bfloat16)
    assert ((out[:T].double() - packed.double()).abs() <= 2 * bound).all() and ((lse2[:T].double() - lse.double()).abs() <= 2 * lse_bound).all()
    assert (out[T:] == 7.0).all() and (lse2[T:] == 7.0).all()


def test_same_page_twice():
    """Sequences that share the pages of a common beginning, and a table that names one page twice."""
    b = batch(27, torch.bfloat16, [64, 64, 96], [1, 40, 2], 4, 2, 128, 32)
    b["table"][1, :2] = b["table"][0, :2]
    b["table"][2, 1] = b["table"][2, 0]
    check(b, 0.1, torch.bfloat16)


@pytest.mark.parametrize("H_q,H_kv,d,dtype", [(4, 2, 128, torch.bfloat16), (2, 2, 64, torch.bfloat16), (4, 1, 128, torch.float32)])
def test_pools_beyond_32_bit_offsets(H_q, H_kv, d, dtype):
    """Pages more than 4 GiB into their pools give what the same pages give at the front."""
    news, lens, page = [1, 90, 3], [150, 40, 33], 32
    small = batch(28, dtype, lens, news, H_q, H_kv, d, page)
    n = small["k_pool"].shape[0]
    page_bytes = H_kv * page * d * small["k_pool"].element_size()
    far = 2 ** 32 // page_bytes + 5
    big = dict(small)
    for name in ("k_pool", "v_pool"):
        big[name] = torch.zeros((far + n, H_kv, page, d), dtype=dtype, device=DEV)
        big[name][far:] = small[name]
    big["table"] = torch.where(small["table"] >= 0, small["table"] + far, small["table"])
    out, lse = run(small, 0.1)
    out, lse = out.clone(), lse.clone()
    got, got_lse = run(big, 0.1)
    assert torch.equal(got, out) and torch.equal(got_lse, lse)
    sums, kept, pools = [], [], []
    for b in (small, big):
        s = torch.zeros(3, H_kv, b["capacity"], device=DEV)
        M.mcsd_attn_weight_sums(M.weight_sums_args(b["q"], b["k_pool"], b["table"], b["chunk_start"], b["prefix_len"], lse, s, 0.1))
        prefix, keep, flags = b["prefix_len"] + torch.tensor(news, dtype=torch.int32, device=DEV), torch.full((3,), 35, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
        k = torch.zeros(s.shape, dtype=torch.int32, device=DEV)
        M.mcsd_kv_evict_paged(M.evict_args(b["k_pool"], b["v_pool"], b["table"], s, prefix, keep, k, flags, 1, 8))
        rows = torch.randn(2, H_kv, d, generator=gen(29)).to(dtype).to(DEV)
        slots = (b["table"][:2, 1] * page + 7).to(torch.int32)
        if int(slots.max()) < 2 ** 31 - 1:
            M.mcsd_kv_store_paged(M.store_args(rows, rows, slots, b["k_pool"], b["v_pool"]))
        torch.cuda.synchronize()
        assert flags.tolist() == [0, 0, 0]
        sums.append(s), kept.append(k), pools.append(b["k_pool"][-n:])
    assert torch.equal(sums[0], sums[1]) and torch.equal(kept[0], kept[1])
    assert torch.equal(torch.nan_to_num(pools[0].float()), torch.nan_to_num(pools[1].float()))


@pytest.mark.parametrize("shape", [([500, 3, 0, 64], [1, 1, 1, 1], 8, 2, 128), ([300, 2000], [200, 70], 6, 2, 128), ([300, 20], [33, 9], 14, 2, 80),
                                   ([90], [500], 2, 1, 256)])
@pytest.mark.parametrize("last", [0, 1, 40])
def test_weight_sums_of_more_rows(shape, last):
    lens, news, H_q, H_kv, d = shape
    b = batch(30, torch.bfloat16, lens, news, H_q, H_kv, d, 32)
    scale = 1 / math.sqrt(d)
    lse = R.attention(b, scale, torch.bfloat16)[2].float()
    sums = torch.rand(len(lens), H_kv, b["capacity"], generator=gen(31)).to(DEV)
    want, bound = R.weight_sums(b, scale, lse, sums, last)
    M.mcsd_attn_weight_sums(M.weight_sums_args(b["q"], b["k_pool"], b["table"], b["chunk_start"], b["prefix_len"], lse, sums, scale, last))
    torch.cuda.synchronize()
    assert ((sums.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("capacity", [4096, 4128, 8192, 8224, 16384, 16416])
def test_evict_capacities(capacity):
    """Around the lengths where the selection takes more threads, and where a row no longer fits their registers."""
    evict_case([capacity, capacity - 1, 3], [capacity // 2, capacity - 2, 2], 4, 33, None, 2, 16, torch.bfloat16, 32, False, some_zero, capacity=capacity)


def test_one_sequence_evicted_again_and_again():
    """Down to one row; what the sums and positions say follows the rows."""
    d, page, n = 64, 32, 200
    g = gen(32)
    k = torch.randn(8, 1, page, d, generator=g).to(torch.bfloat16).to(DEV)
    v = torch.randn(8, 1, page, d, generator=g).to(torch.bfloat16).to(DEV)
    table = torch.randperm(8, generator=g)[:7].int().view(1, 7).to(DEV)
    sums = torch.rand(1, 1, 224, generator=g).to(DEV)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    prefix, flags, kept = i32([n]), i32([0]), i32([[[0] * 224]])
    rows, s = R.rows_of(k, table[0], page, n)[0], sums[0, 0, :n].clone()
    for keep in (199, 150, 150, 64, 33, 32, 5, 1):
        M.mcsd_kv_evict_paged(M.evict_args(k, v, table, sums, prefix, i32([keep]), kept, flags, 1, 2))
        torch.cuda.synchronize()
        at = R.evicted(len(s), keep, 1, 2, s.tolist())
        rows, s = rows[at], s[at]
        assert int(prefix) == keep and kept[0, 0, :keep].tolist() == at
        assert torch.equal(sums[0, 0, :keep], s) and torch.equal(R.rows_of(k, table[0], page, keep)[0], rows)


WIDE = [  # enough work for the kernel that takes 256 rows a workgroup: (lens, news, H_q, H_kv, page)
    ([0], [700], 64, 64, 64),
    ([0], [257], 256, 256, 32),
    ([63], [257], 256, 128, 32),
    ([31, 500, 0], [300, 1, 513], 128, 64, 96),
    ([5000], [100], 64, 8, 128),
    ([5000, 40, 1], [70, 100, 60], 128, 16, 64),
    ([1, 2, 3], [22, 129, 400], 384, 128, 32),
    ([2000, 2016, 2017], [96, 96, 96], 56, 8, 32),
    ([3000], [64], 256, 16, 32),
    ([10, 0, 900], [0, 300, 65], 96, 96, 160),
]


@pytest.mark.parametrize("shape", WIDE)
def test_wide(shape):
    lens, news, H_q, H_kv, page = shape
    check(batch(33, torch.bfloat16, lens, news, H_q, H_kv, 128, page), 1 / math.sqrt(128), torch.bfloat16)


@pytest.mark.parametrize("scale", [0.0, 1.0])
def test_wide_scale(scale):
    check(batch(34, torch.bfloat16, [100, 0], [300, 270], 128, 128, 128, 64), scale, torch.bfloat16)


@pytest.mark.parametrize("lens,news,H_kv", [([70], [300], 128), ([2500], [280], 16)])
def test_wide_no_number(lens, news, H_kv):
    """Before, inside and behind the tiles that rows see in part, keys in one piece and cut; and in the keys themselves."""
    b = batch(35, torch.bfloat16, lens, news, H_kv, H_kv, 128, 32)
    L, n = lens[0], news[0]
    clean, clean_lse = run(b, 0.1)
    clean, clean_lse = clean.clone(), clean_lse.clone()
    for pos in (30, L - 1, L + 5, L + 130, L + n - 1):
        page, row = int(b["table"][0, pos // 32]), pos % 32
        old = b["v_pool"][page, :, row].clone()
        b["v_pool"][page, 0, row, 7], b["v_pool"][page, 1, row, 9] = float("nan"), -float("inf")
        out, lse = run(b, 0.1)
        first = max(0, pos - L)
        want = clean.clone()
        want[first:, 0, 7], want[first:, 1, 9] = float("nan"), -float("inf")
        assert torch.equal(lse, clean_lse) and torch.equal(torch.nan_to_num(out.float(), nan=1e30), torch.nan_to_num(want.float(), nan=1e30))
        b["v_pool"][page, :, row] = old
    page, row = int(b["table"][0, (L + 50) // 32]), (L + 50) % 32
    b["k_pool"][page, :, row] = float("nan")
    out, lse = run(b, 0.1)
    assert torch.equal(out[:50], clean[:50]) and torch.equal(lse[:50], clean_lse[:50]) and torch.isnan(lse[50:]).all()


def test_wide_bad_pages():
    b = batch(36, torch.bfloat16, [100, 64], [300, 200], 128, 64, 128, 32)
    b["table"][0, 1], b["table"][0, 5], b["table"][1, 0], b["table"][1, 7] = -1, 2 ** 31 - 1, b["k_pool"].shape[0], -2 ** 31
    check(b, 0.1, torch.bfloat16)


def test_wide_lengths_beyond_the_capacity():
    b = batch(37, torch.bfloat16, [200], [312], 64, 64, 128, 32)
    below, bound, _, _ = R.attention(b, 0.1, torch.bfloat16)
    b["capacity"] = 416
    out, _ = run(b, 0.1)
    assert ((out.double() - below).abs() <= bound)[:216].all()         # (not to the bit: fewer keys may be cut elsewhere)
    v = R.rows_of(b["v_pool"], b["table"][0], 32, 416)
    k = R.rows_of(b["k_pool"], b["table"][0], 32, 416)
    want = torch.softmax(torch.einsum("thd,hkd->thk", b["q"][216:].double(), k) * 0.1, -1)
    want = torch.einsum("thk,hkd->thd", want, v)
    assert (out[216:].double() - want).abs().max() < 2.0 ** -7 * 4


@pytest.mark.parametrize("layers,keeps", [(40, [300, 150, 7]), (40, [999, 999, 999]), (3, [300, 999, 150])])
def test_evict_many_heads(layers, keeps):
    """More heads than workgroups at once; sequences that keep everything among others."""
    evict_case([700, 300, 40], keeps, 4, 9, layers, 6, 128, torch.bfloat16, 32, False, some_zero)


def test_evict_lengths_out_of_range():
    """prefix_len below 0 counts as 0, beyond the capacity as that, and becomes what is kept."""
    k = torch.randn(6, 1, 32, 64, generator=gen(38)).to(torch.bfloat16).to(DEV)
    before = k.clone()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    prefix, flags, kept = i32([-5, 2 ** 31 - 1]), i32([9, 9]), torch.full((2, 1, 64), -7, dtype=torch.int32, device=DEV)
    sums = torch.arange(128.0, device=DEV).view(2, 1, 64).contiguous()
    M.mcsd_kv_evict_paged(M.evict_args(k, k.clone(), i32([[0, 1], [2, 3]]), sums, prefix, i32([10, 32]), kept, flags, 0, 0))
    torch.cuda.synchronize()
    assert prefix.tolist() == [0, 32] and flags.tolist() == [0, 0] and (kept[0] == -7).all() and kept[1, 0, :32].tolist() == list(range(32, 64))
    assert torch.equal(k[2], before[3]) and torch.equal(k[:2], before[:2]) and torch.equal(k[3:], before[3:])
