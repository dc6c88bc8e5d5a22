"""Chunk attention's kernel for many rows, with shapes that it takes: every test looks at what the launch left in the workspace's last 256 bytes (items of
this kernel that were taken; rows beyond which a sequence belongs to it) and so shows that it ran, or that the device decided against it."""
import math

import pytest
import torch

from paper_2401_06706_amd import binding as M
from tests import chunk_ref as R
from tests.test_gpu_chunk import DEV, gen

pytestmark = pytest.mark.gpu
SCALE = 0.09
NEVER = 0x7fffffff


def batch(seed, lens, news, H_q, H_kv, page=32):
    return R.make_batch(gen(seed), DEV, torch.bfloat16, lens, news, H_q, H_kv, 128, page)


def run(b):
    """out, lse, (items taken, rows beyond which a sequence belongs to the kernel for many)"""
    q = b["q"]
    out, lse = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV), torch.full(q.shape[:2], 7.0, device=DEV)
    need = M.mcsd_chunk_workspace_bytes(M.chunk_desc(q, b["k_pool"], b["table"], SCALE, b["capacity"]))
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device=DEV)
    args = M.chunk_attn_args(q, b["k_pool"], b["v_pool"], b["table"], b["chunk_start"], b["prefix_len"], out, SCALE, b["capacity"], lse, ws)
    M.mcsd_kernel_timing(True)
    M.mcsd_chunk_attn_paged(args)
    torch.cuda.synchronize()
    launched = M.mcsd_kernel_timing_read()["chunk_wide"][1]
    M.mcsd_kernel_timing(False)
    assert launched == 1
    return out, lse, tuple(ws[need - 256:].view(torch.int32)[:2].tolist())


def check(b, wide=True):
    out, lse, (taken, many) = run(b)
    assert (taken > 0 and many < NEVER) if wide else (taken == 0 and many == NEVER)
    want, bound, want_lse, lse_bound = R.attention(b, SCALE, torch.bfloat16)
    err = (out.double() - want).abs()
    assert (err <= bound).all(), f"{float((err - bound).max())} over at {torch.nonzero(~(err <= bound))[:4].tolist()}"
    assert ((lse.double() - want_lse).abs() <= lse_bound).all()


@pytest.mark.parametrize("heads", [32, 64])
def test_more_pages_than_lanes(heads):
    """Items of 68 and 135 pages, of which a workgroup holds 64 entries at a time; again where what is no number has an item done twice."""
    b = batch(51, [8000, 7000], [600, 600], heads, heads)
    check(b)
    clean, clean_lse, _ = run(b)
    for pos in (8000 + 300, 8000 + 599, 4000):
        page, row = int(b["table"][0, pos // 32]), pos % 32
        old = b["v_pool"][page, :, row].clone()
        b["v_pool"][page, 0, row, 7], b["v_pool"][page, 1, row, 9] = float("nan"), -math.inf
        out, lse, _ = run(b)
        want, first = clean.clone(), max(0, pos - 8000)
        want[first:600, 0, 7], want[first:600, 1, 9] = float("nan"), -math.inf
        assert torch.equal(lse, clean_lse) and torch.equal(torch.nan_to_num(out.float(), nan=1e30), torch.nan_to_num(want.float(), nan=1e30))
        b["v_pool"][page, :, row] = old


@pytest.mark.parametrize("B,long,far", [(70, 130, {66: 6000}), (140, 70, {66: 6000, 132: 9000}), (300, 40, {})])
def test_more_sequences_than_lanes(B, long, far):
    """Sequences of many rows among the first 64 and behind them, cut and whole, beside decoding ones and ones without new tokens."""
    lens = [far.get(b, (53 * b) % 400) for b in range(B)]
    news = [0 if b % 6 == 5 else 1 if b % 3 == 1 else long for b in range(B)]
    check(batch(52, lens, news, 32, 8))


@pytest.mark.parametrize("news,wide", [([1] * 5 + [200], False), ([1] * 5 + [400], True), ([1] * 5 + [900], True)])
def test_the_device_decides(news, wide):
    """One prompt among decoding sequences: they have most of the work, or it has."""
    check(batch(53, [3000] * 5 + [4000], news, 32, 16, 64), wide)


@pytest.mark.parametrize("heads,L,n,capacity", [(128, 200, 312, 416), (32, 2000, 700, 2304), (256, 300, 300, 576)])
def test_lengths_beyond_the_capacity(heads, L, n, capacity):
    """Keys in one piece and cut; rows past the capacity see what lies below it."""
    b = batch(54, [L], [n], heads, heads)
    want, bound, want_lse, lse_bound = R.attention(b, SCALE, torch.bfloat16)
    fit, beyond = capacity - L, L + n - capacity
    # a row past the capacity is a token at its last position
    last = dict(b, lens=[capacity - 1] * beyond, news=[1] * beyond, start=list(range(beyond + 1)), q=b["q"][fit:], table=b["table"].expand(beyond, -1))
    for x, y in zip((want, bound, want_lse, lse_bound), R.attention(last, SCALE, torch.bfloat16)):
        x[fit:] = y
    b["capacity"] = capacity
    out, lse, (taken, _) = run(b)
    assert taken > 0
    assert ((out.double() - want).abs() <= bound).all() and ((lse.double() - want_lse).abs() <= lse_bound).all()


def test_no_number_in_cut_keys():
    """Before, inside and behind the tiles that rows see in part, where several workgroups share a row's keys."""
    b = batch(55, [2500], [280], 32, 32)
    clean, clean_lse, (taken, _) = run(b)
    assert taken > 0
    for pos in (30, 2499, 2505, 2630, 2779):
        page, row = int(b["table"][0, pos // 32]), pos % 32
        old = b["v_pool"][page, :, row].clone()
        b["v_pool"][page, 0, row, 7], b["v_pool"][page, 1, row, 9] = float("nan"), -math.inf
        out, lse, _ = run(b)
        want, first = clean.clone(), max(0, pos - 2500)
        want[first:, 0, 7], want[first:, 1, 9] = float("nan"), -math.inf
        assert torch.equal(lse, clean_lse) and torch.equal(torch.nan_to_num(out.float(), nan=1e30), torch.nan_to_num(want.float(), nan=1e30))
        b["v_pool"][page, :, row] = old


@pytest.mark.parametrize("shape", [([70], [300], 256, 256), ([31, 500, 0], [300, 1, 513], 128, 64), ([0], [700], 64, 64)])
def test_bad_pages(shape):
    lens, news, H_q, H_kv = shape
    b = batch(56, lens, news, H_q, H_kv)
    b["table"][0, 1], b["table"][0, 5], b["table"][0, 7] = -1, 2 ** 31 - 1, b["k_pool"].shape[0]
    check(b)


# ---- calls one after the other: the counter of items has to start from 0 in every launch and replay
T_MAX, CAPACITY, PAGE, N_PAGES = 700, 4096, 32, 400
ROUNDS = [([2500, 40, 900], [280, 1, 300], True), ([40, 0, 10], [70, 1, 1], False), ([3500, 3000, 100], [1, 400, 90], True), ([3000, 100, 2000], [1, 1, 1], False),
          ([3900, 50, 7], [100, 0, 65], True), ([0, 10, 700], [256, 200, 244], False)]


class Batch:
    def __init__(self, H_q, H_kv, ws=None):
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
        new = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=DEV)
        g = gen(57)
        self.k_pool, self.v_pool = (torch.randn(N_PAGES, H_kv, PAGE, 128, generator=g).bfloat16().to(DEV) for _ in range(2))
        self.table = torch.randperm(N_PAGES, generator=g)[:3 * CAPACITY // PAGE].int().view(3, -1).to(DEV)
        self.q, self.out, self.lse = new(T_MAX, H_q, 128), new(T_MAX, H_q, 128), torch.zeros(T_MAX, H_q, device=DEV)
        self.start, self.prefix = i32([0] * 4), i32([0] * 3)
        need = M.mcsd_chunk_workspace_bytes(M.chunk_desc(self.q, self.k_pool, self.table, SCALE, CAPACITY))
        self.ws = torch.full((need,), 0xff, dtype=torch.uint8, device=DEV) if ws is None else ws
        self.args = M.chunk_attn_args(self.q, self.k_pool, self.v_pool, self.table, self.start, self.prefix, self.out, SCALE, CAPACITY, self.lse, self.ws)

    def feed(self, r):
        lens, news, _ = ROUNDS[r]
        self.prefix.copy_(torch.tensor(lens, dtype=torch.int32))
        self.start.copy_(torch.tensor([sum(news[:b]) for b in range(4)], dtype=torch.int32))
        self.q.copy_(torch.randn(*self.q.shape, generator=gen(60 + r)).bfloat16())
        self.out.fill_(7.0)
        self.lse.fill_(7.0)

    def state(self):
        return self.out.clone().view(torch.int16), self.lse.clone().view(torch.int32)

    def taken(self):
        return int(self.ws[-256:].view(torch.int32)[0])


def eager(heads):
    one, states = Batch(*heads), []
    for r, (lens, news, wide) in enumerate(ROUNDS):
        one.feed(r)
        M.mcsd_chunk_attn_paged(one.args)
        torch.cuda.synchronize()
        assert (one.taken() > 0) == wide, r
        states.append(one.state())
    return states


def same(got, want, r):
    assert all(torch.equal(x, y) for x, y in zip(got, want)), r


def test_rounds_against_the_definition():
    one = Batch(64, 32)
    for r, (lens, news, wide) in enumerate(ROUNDS):
        one.feed(r)
        M.mcsd_chunk_attn_paged(one.args)
        torch.cuda.synchronize()
        b = {"lens": lens, "news": news, "start": one.start.tolist(), "q": one.q, "k_pool": one.k_pool, "v_pool": one.v_pool, "table": one.table, "page": PAGE}
        want, bound, want_lse, lse_bound = R.attention(b, SCALE, torch.bfloat16)
        T = sum(news)
        assert ((one.out.double() - want).abs() <= bound)[:T].all() and ((one.lse.double() - want_lse).abs() <= lse_bound)[:T].all()
        assert (one.out[T:] == 7.0).all() and (one.lse[T:] == 7.0).all() and (one.taken() > 0) == wide


@pytest.mark.parametrize("heads", [(64, 64), (64, 32), (64, 16)])
def test_two_graphs_share_a_workspace(heads):
    """Replayed in turn with new lengths each time, so that the device decides anew; the workspace filled with rubbish, and eager calls in it, between the replays."""
    want = eager(heads)
    first = Batch(*heads)
    batches, graphs, other = [first, Batch(*heads, ws=first.ws)], [], Batch(*heads, ws=first.ws)
    for b in batches:
        b.feed(0)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            M.mcsd_chunk_attn_paged(b.args)
    for r in [0, 1, 2, 3, 4, 5, 0, 2, 4]:
        for b, graph in zip(batches, graphs):
            b.feed(r)
            graph.replay()
        torch.cuda.synchronize()
        assert (first.taken() > 0) == ROUNDS[r][2]
        for b in batches:
            same(b.state(), want[r], r)
        first.ws.fill_(0xff)
        other.feed((r + 1) % 6)
        M.mcsd_chunk_attn_paged(other.args)
        torch.cuda.synchronize()
        same(other.state(), want[(r + 1) % 6], r)


def test_two_streams():
    """Side by side, each with its own workspace."""
    heads = (64, 32)
    want, batches, streams = eager(heads), [Batch(*heads), Batch(*heads)], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for r in range(len(ROUNDS)):
        for i, (b, stream) in enumerate(zip(batches, streams)):
            with torch.cuda.stream(stream):
                b.feed((r + i) % len(ROUNDS))
                M.mcsd_chunk_attn_paged(b.args, stream)
        torch.cuda.synchronize()
        for i, b in enumerate(batches):
            same(b.state(), want[(r + i) % len(ROUNDS)], r)
