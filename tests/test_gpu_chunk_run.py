"""Pages, store, chunk attention, weight sums, eviction, tree attention and log probabilities one after the other, as a serving loop
makes them: eagerly against the definitions at every call, captured and replayed against the eager run, on other streams, side by side."""
import math

import pytest
import torch

from paper_2401_06706_amd import binding as M
from tests import chunk_ref as R
from tests.test_gpu_chunk import DEV, gen

pytestmark = pytest.mark.gpu

B, H_q, H_kv, D, PAGE, N_PAGES, WIDTH, T_MAX, N_TREE, VOCAB, N_TOP = 3, 8, 2, 128, 32, 40, 8, 200, 4, 515, 3
SCALE = 1 / math.sqrt(D)
ROUNDS = [[40, 1, 130], [1, 1, 1], [1, 70, 0], [1, 1, 1], [90, 1, 1]]       # new tokens per sequence
PARENT = [-1, 0, 0, 1]


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Loop:
    """State of a batch and the calls of one round over it."""

    def __init__(self, dtype=torch.bfloat16):
        self.dtype = dtype
        new = lambda *s: torch.zeros(*s, dtype=dtype, device=DEV)
        self.k_pool, self.v_pool = new(N_PAGES, H_kv, PAGE, D), new(N_PAGES, H_kv, PAGE, D)
        self.prefix, self.want, self.held, self.flags = i32([0] * B), i32([0] * B), i32([0] * B), i32([0] * B)
        self.table, self.free, self.n_free = i32([[-1] * WIDTH] * B), i32(list(range(N_PAGES))), i32([N_PAGES])
        self.start, self.slots = i32([0] * (B + 1)), i32([-1] * T_MAX)
        self.q, self.k, self.v = new(T_MAX, H_q, D), new(T_MAX, H_kv, D), new(T_MAX, H_kv, D)
        self.out, self.lse = new(T_MAX, H_q, D), torch.zeros(T_MAX, H_q, device=DEV)
        self.sums = torch.zeros(B, H_kv, WIDTH * PAGE, device=DEV)
        self.keep, self.kept, self.evict_flags = i32([64, 96, 100]), i32([[[0] * (WIDTH * PAGE)] * H_kv] * B), i32([0] * B)
        self.q_tree, self.k_tree, self.v_tree = new(B, N_TREE, H_q, D), new(B, H_kv, N_TREE, D), new(B, H_kv, N_TREE, D)
        self.tree_out, self.parent = new(B, N_TREE, H_q, D), i32(PARENT)
        self.logits, self.tokens = torch.zeros(B * N_TREE, VOCAB, device=DEV), i32([0] * (B * N_TREE))
        rows = B * N_TREE
        self.logprob, self.entropy = torch.zeros(rows, device=DEV), torch.zeros(rows, device=DEV)
        self.rank, self.logit_flags, self.top = i32([0] * rows), i32([0] * rows), i32([[0] * N_TOP] * rows)
        self.top_lp = torch.zeros(rows, N_TOP, device=DEV)
        cap = WIDTH * PAGE
        page_args = lambda want: M.page_args(self.prefix, want, self.held, self.table, self.free, self.n_free, self.flags, PAGE, self.start, self.slots)
        need = M.mcsd_chunk_workspace_bytes(M.chunk_desc(self.q, self.k_pool, self.table, SCALE, cap))
        self.ws = torch.full((max(need, 1),), 0xff, dtype=torch.uint8, device=DEV)
        tree_desc = M.attn_desc(B, N_TREE, H_q, H_kv, D, M.DTYPE_FP32 if dtype == torch.float32 else M.DTYPE_BF16, cap, SCALE)
        self.tree_ws = torch.zeros(max(1, M.mcsd_attn_workspace_bytes(tree_desc)), dtype=torch.uint8, device=DEV)
        self.assign, self.release = page_args(self.want), page_args(self.prefix)
        self.store = M.store_args(self.k, self.v, self.slots, self.k_pool, self.v_pool)
        self.attend = M.chunk_attn_args(self.q, self.k_pool, self.v_pool, self.table, self.start, self.prefix, self.out, SCALE, cap, self.lse,
                                        self.ws if need else None)
        self.weigh = M.weight_sums_args(self.q, self.k_pool, self.table, self.start, self.prefix, self.lse, self.sums, SCALE, 4)
        self.evict = M.evict_args(self.k_pool, self.v_pool, self.table, self.sums, self.prefix, self.keep, self.kept, self.evict_flags, 4, 16)
        self.tree, self.tree_pages = M.paged_attn_args(self.q_tree, self.k_pool, self.v_pool, self.table, self.prefix, self.k_tree, self.v_tree,
                                                       self.parent, self.tree_out, SCALE, cap, self.tree_ws)
        self.answer = M.logprob_args(self.logits, self.tokens, self.logprob, self.entropy, self.rank, self.top, self.top_lp, self.logit_flags)

    def feed(self, r):
        """The inputs of round r."""
        g = gen(100 + r)
        news = ROUNDS[r % len(ROUNDS)]
        self.want.copy_(self.prefix + i32(news))
        for t in (self.q, self.k, self.v, self.q_tree, self.k_tree, self.v_tree):
            t.copy_(torch.randn(*t.shape, generator=g).to(self.dtype))
        self.logits.copy_(3 * torch.randn(*self.logits.shape, generator=g))
        self.tokens.copy_(torch.randint(0, VOCAB, self.tokens.shape, generator=g).int())
        for t in (self.out, self.lse):
            t.fill_(7.0)
        return news

    def calls(self, stream=None, check=lambda name: None):
        M.mcsd_page_assign(self.assign, stream)
        M.mcsd_kv_store_paged(self.store, stream)
        M.mcsd_chunk_attn_paged(self.attend, stream)
        check("attend")
        M.mcsd_attn_weight_sums(self.weigh, stream)
        check("weigh")
        self.prefix.copy_(self.want)
        M.mcsd_kv_evict_paged(self.evict, stream)
        check("evict")
        M.mcsd_page_assign(self.release, stream)
        M.mcsd_tree_attn_paged(self.tree, self.tree_pages, stream)
        check("tree")
        M.mcsd_token_logprobs(self.answer, stream)
        check("answer")

    def state(self):
        return [t.clone() for t in (self.out, self.lse, self.sums, self.kept, self.evict_flags, self.prefix, self.held, self.table, self.n_free, self.k_pool,
                                    self.v_pool, self.tree_out, self.logprob, self.entropy, self.rank, self.logit_flags, self.top, self.top_lp, self.flags)]


def same(a, b):
    for x, y in zip(a, b):
        bits = lambda t: t if t.dtype == torch.int32 else t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)
        assert torch.equal(bits(x), bits(y))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rounds(dtype):
    loop = Loop(dtype)
    for r in range(len(ROUNDS)):
        lens, news = loop.prefix.tolist(), loop.feed(r)
        T = sum(news)
        batch = {"lens": lens, "news": news, "start": [sum(news[:b]) for b in range(B + 1)], "q": loop.q, "page": PAGE}
        old_sums = loop.sums.clone()

        def check(name):
            torch.cuda.synchronize()
            batch.update(k_pool=loop.k_pool, v_pool=loop.v_pool, table=loop.table)
            if name == "attend":
                assert loop.start.tolist() == batch["start"] and loop.flags.tolist() == [0] * B
                want, bound, want_lse, lse_bound = R.attention(batch, SCALE, dtype)
                assert ((loop.out.double() - want).abs() <= bound)[:T].all() and ((loop.lse.double() - want_lse).abs() <= lse_bound)[:T].all()
                assert (loop.out[T:] == 7.0).all() and (loop.lse[T:] == 7.0).all()
                for b in range(B):          # what was stored is what stands behind the cached rows
                    k = R.rows_of(loop.k_pool, loop.table[b], PAGE, lens[b] + news[b])[:, lens[b]:]
                    assert torch.equal(k, loop.k[batch["start"][b]:batch["start"][b + 1]].double().transpose(0, 1))
            if name == "weigh":
                want, bound = R.weight_sums(batch, SCALE, loop.lse, old_sums, 4)
                assert ((loop.sums.double() - want).abs() <= bound).all()
                batch["before"] = (loop.sums.clone(), [R.rows_of(loop.k_pool, loop.table[b], PAGE, lens[b] + news[b]) for b in range(B)])
            if name == "evict":
                sums, rows = batch["before"]
                assert loop.evict_flags.tolist() == [0] * B
                for b in range(B):
                    n, keep = lens[b] + news[b], int(loop.keep[b])
                    m = min(n, keep)
                    assert int(loop.prefix[b]) == m
                    for h in range(H_kv):
                        kept = R.evicted(n, keep, 4, 16, sums[b, h].tolist())
                        assert loop.kept[b, h, :m].tolist() == kept and torch.equal(loop.sums[b, h, :m], sums[b, h, kept])
                        assert torch.equal(R.rows_of(loop.k_pool, loop.table[b], PAGE, m)[h], rows[b][h, kept])
            if name == "tree":
                assert loop.held.tolist() == [-(-int(n) // PAGE) for n in loop.prefix] and int(loop.n_free) == N_PAGES - int(loop.held.sum())
                for b in range(B):
                    n = int(loop.prefix[b])
                    k, v = (R.rows_of(p, loop.table[b], PAGE, n) for p in (loop.k_pool, loop.v_pool))
                    for i in range(N_TREE):
                        line, at = [], i
                        while at >= 0:
                            line.insert(0, at)
                            at = PARENT[at]
                        for head in range(H_q):
                            g = head // (H_q // H_kv)
                            kk = torch.cat([k[g], loop.k_tree[b, g, line].double()])
                            vv = torch.cat([v[g], loop.v_tree[b, g, line].double()])
                            p = torch.softmax(kk @ loop.q_tree[b, i, head].double() * SCALE, 0)
                            mass = p @ vv.abs()             # weights and the result rounded once each, and 2^-12 for fp32 arithmetic over 300 keys
                            step = 2 * 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
                            assert ((loop.tree_out[b, i, head].double() - p @ vv).abs() <= (step + 2.0 ** -12) * mass).all()
            if name == "answer":
                assert loop.logit_flags.tolist() == [0] * (B * N_TREE)
                for i in range(B * N_TREE):
                    lp, entropy, rank, ids, lps = R.logprobs(loop.logits[i].cpu(), int(loop.tokens[i]), 1.0, N_TOP)
                    assert int(loop.rank[i]) == rank and loop.top[i].tolist() == ids
                    spread = float(loop.logits[i].max() - loop.logits[i].min())
                    for got, want in [(loop.logprob[i], lp), (loop.entropy[i], entropy)] + list(zip(loop.top_lp[i], lps)):
                        assert abs(float(got) - want) <= R.logprob_bound(VOCAB, want, 2 * spread)

        loop.calls(check=check)


def eager_states(rounds):
    loop, states = Loop(), []
    for r in range(rounds):
        loop.feed(r)
        loop.calls()
        torch.cuda.synchronize()
        states.append(loop.state())
    return states


def test_captured_and_replayed():
    """A round in a graph goes on from the state of the last one; eager rounds of another batch between the replays."""
    want = eager_states(7)
    loop, other = Loop(), Loop()
    saved = loop.state()
    loop.feed(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        loop.calls(side)
    torch.cuda.synchronize()
    same(loop.state()[2:], saved[2:])                   # (capturing runs nothing)
    for r in range(7):
        loop.feed(r)
        graph.replay()
        other.feed(r)
        other.calls()
        torch.cuda.synchronize()
        same(loop.state(), want[r])
        same(other.state(), want[r])


def test_two_batches_on_two_streams():
    """Each with its own workspace: neither waits for the other, none disturbs the other."""
    want = eager_states(5)
    loops, streams = [Loop(), Loop()], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for r in range(5):
        for loop, stream in zip(loops, streams):
            with torch.cuda.stream(stream):
                loop.feed(r)
                loop.calls(stream)
        torch.cuda.synchronize()
        for loop in loops:
            same(loop.state(), want[r])


def test_two_graphs_share_a_workspace():
    """One after the other on one stream, replayed in turn: a workspace holds nothing from call to call."""
    loops = [Loop(), Loop()]
    loops[1].ws = loops[0].ws
    need = loops[0].ws.numel()
    cap = WIDTH * PAGE
    loops[1].attend = M.chunk_attn_args(loops[1].q, loops[1].k_pool, loops[1].v_pool, loops[1].table, loops[1].start, loops[1].prefix, loops[1].out, SCALE,
                                        cap, loops[1].lse, loops[0].ws if need > 1 else None)
    want = eager_states(4)
    graphs = []
    for loop in loops:
        loop.feed(0)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            loop.calls()
    for r in range(4):
        for loop, graph in zip(loops, graphs):
            loop.feed(r)
            graph.replay()
        loops[0].ws.fill_(0xff)
        torch.cuda.synchronize()
        for loop in loops:
            same(loop.state(), want[r])
