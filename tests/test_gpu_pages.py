"""Block tables, slot maps and the free list on the GPU against a sequential account of the same rules."""
import numpy as np
import pytest
import torch

from paper_2401_06706_amd import binding as M

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def account(prefix, want, held, table, free, n_free, ps, n_pages, max_slots):
    """The header's rules, one page after the other."""
    B, width = table.shape
    held, table, free = held.copy(), table.copy(), free.copy()
    n_free = min(max(int(n_free), 0), n_pages)
    flags = np.zeros(B, np.int64)
    need = np.zeros(B, np.int64)
    for b in range(B):
        need[b] = held[b]
        if want[b] < 0 or prefix[b] < 0 or not 0 <= held[b] <= width:
            flags[b] = 512
        elif -(-int(want[b]) // ps) > width:
            flags[b] = 256
        else:
            need[b] = -(-int(want[b]) // ps)
    ok = flags == 0
    stack = list(free[:n_free])
    owner = [-1] * n_free
    for b in range(B - 1, -1, -1):
        if ok[b]:
            for c in range(held[b] - 1, need[b] - 1, -1):
                stack.append(table[b, c])
                owner.append(b)
                table[b, c] = -1
    for b in owner[n_pages:]:
        flags[b] |= 512
    stack = stack[:n_pages]
    free[:len(stack)] = stack
    top, asked, slots, start = len(stack), 0, [], [0]
    for b in range(B):
        lack = max(0, need[b] - held[b]) if ok[b] else 0
        asked += lack
        served = ok[b] and (lack == 0 or asked <= top)
        if served:
            for c in range(held[b], need[b]):
                table[b, c] = stack.pop()
            held[b] = need[b]
            new = [(int(table[b, i // ps]) * ps + i % ps) if 0 <= table[b, i // ps] < n_pages else -1 for i in range(prefix[b], want[b])]
            slots += new
            if new and len(slots) > max_slots:
                flags[b] |= 1024
        elif ok[b]:
            flags[b] |= 256
        start.append(min(len(slots), max_slots))
    slot_map = (slots + [-1] * max_slots)[:max_slots]
    return dict(table=table, held=held, free=free, n_free=np.array([len(stack)]), flags=flags, start=np.array(start), slots=np.array(slot_map))


def run(prefix, want, held, table, free, n_free, ps, max_slots, maps=True):
    t = dict(held=i32(held), table=i32(table), free=i32(free), n_free=i32([n_free]), flags=i32(np.full(len(prefix), 77)))
    if maps:
        t.update(start=i32(np.full(len(prefix) + 1, -9)), slots=i32(np.full(max_slots, -9)))
    args = M.page_args(i32(prefix), i32(want), t["held"], t["table"], t["free"], t["n_free"], t["flags"], ps, t.get("start"), t.get("slots"))
    M.mcsd_page_assign(args)
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in t.items()}, t, args


def same(got, want):
    for k, v in got.items():
        assert (v == want[k]).all(), (k, v[v != want[k]][:5], want[k][v != want[k]][:5])


def state(rng, B, ps, most, spare):
    """A pool in use: lengths, pages held, a table and a free stack in random order."""
    prefix = rng.integers(0, most + 1, size=B)
    held = -(-prefix // ps) + rng.integers(0, 2, size=B)
    width = int(max(held.max(), -(-2 * most // ps), 1))
    n_pages = int(held.sum()) + spare
    order = rng.permutation(n_pages)
    table, at = np.full((B, width), -1), 0
    for b in range(B):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
    free = np.full(n_pages, -3)
    free[:spare] = order[at:]
    return prefix, held, table, free, n_pages


@pytest.mark.parametrize("B,ps,most,spare,max_slots", [(1, 32, 1, 1, 4), (1, 64, 500, 0, 7), (5, 1, 20, 9, 100), (16, 64, 4096, 12, 400), (63, 32, 300, 40, 1),
                                                       (64, 96, 300, 400, 5000), (65, 32, 33, 20, 2000), (1000, 64, 2000, 3000, 60000),
                                                       (1025, 32, 100, 90, 20000), (3000, 16, 50, 4000, 40000)])
def test_against_the_account(B, ps, most, spare, max_slots):
    rng = np.random.default_rng(B + ps)
    prefix, held, table, free, n_pages = state(rng, B, ps, most, spare)
    want = prefix + rng.integers(0, 9, size=B)
    new = rng.random(B) < 0.2
    want[new] = rng.integers(0, 2 * most + 1, size=new.sum())
    want[rng.random(B) < 0.15] = 0
    want[rng.random(B) < 0.03] = table.shape[1] * ps + 1          # does not fit its table
    if B > 8:
        prefix[3], want[4], held[5], held[6] = -1, -2, -1, table.shape[1] + 1
    got, _, _ = run(prefix, want, held, table, free, spare, ps, max_slots)
    same(got, account(prefix, want, held, table, free, spare, ps, n_pages, max_slots))


def test_first_that_does_not_fit_stops_those_behind_it():
    z = np.zeros(4, np.int64)
    table, free = np.full((4, 8), -1), np.arange(10)
    # 300 tokens are ten pages, more than a table of eight: that sequence does not count, and the next takes its page
    got, _, _ = run(z, [64, 300, 32, 0], z, table, free, 5, 32, 0, maps=False)
    assert got["held"].tolist() == [2, 0, 1, 0] and got["flags"].tolist() == [0, 256, 0, 0] and got["n_free"][0] == 2
    assert got["table"][0].tolist() == [4, 3] + [-1] * 6 and got["table"][2].tolist() == [2] + [-1] * 7
    # 200 are seven, which the stack does not have: nothing for those behind either
    got, _, _ = run(z, [64, 200, 32, 0], z, table, free, 5, 32, 0, maps=False)
    assert got["held"].tolist() == [2, 0, 0, 0] and got["flags"].tolist() == [0, 256, 256, 0] and got["n_free"][0] == 3


def test_giving_back_restores_the_stack():
    rng = np.random.default_rng(2)
    B, ps, n_pages = 40, 32, 900
    z = np.zeros(B, np.int64)
    free = rng.permutation(n_pages)
    want = rng.integers(0, 700, size=B)
    got, t, _ = run(z, want, z, np.full((B, 22), -1), free, n_pages, ps, 100)
    M.mcsd_page_assign(M.page_args(i32(z), i32(z), t["held"], t["table"], t["free"], t["n_free"], t["flags"], ps))
    assert (t["free"].cpu().numpy() == free).all() and int(t["n_free"]) == n_pages
    assert (t["table"].cpu().numpy() == -1).all() and (t["held"].cpu().numpy() == 0).all()


@pytest.mark.parametrize("n_free", [-5, 0, 6, 1000])
def test_counts_that_do_not_fit_stay_inside_the_pool(n_free):
    """A table that claims pages which the stack holds already: what comes back past the pool's size is lost and flagged."""
    prefix, want, held = np.array([100, 64]), np.array([0, 10]), np.array([4, 2])
    table, free = np.array([[0, 1, 2, 3], [4, 99, -1, -1]]), np.arange(6)
    got, _, _ = run(prefix, want, held, table, free, n_free, 32, 8)
    same(got, account(prefix, want, held, table, free, n_free, 32, 6, 8))


def test_pages_in_a_graph():
    """Replayed: every replay goes on from the state of the last one, as a decode loop does."""
    B, ps, n_pages = 3, 32, 30
    prefix, want = i32([0, 5, 40]), i32([0, 0, 0])
    held, table, free, n_free = i32([0, 0, 0]), i32(np.full((B, 10), -1)), i32(np.arange(n_pages)), i32([n_pages])
    flags, start, slots = i32([0] * B), i32([0] * (B + 1)), i32([0] * 64)
    args = M.page_args(prefix, want, held, table, free, n_free, flags, ps, start, slots)
    M.mcsd_page_assign(args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        M.mcsd_page_assign(args)
    ref = dict(table=table.cpu().numpy(), held=held.cpu().numpy(), free=free.cpu().numpy(), n_free=n_free.cpu().numpy())
    for step, (p, w) in enumerate([([0, 0, 0], [20, 0, 33]), ([20, 0, 33], [33, 300, 40]), ([33, 300, 40], [34, 0, 41]), ([34, 0, 41], [0, 32, 320])]):
        prefix.copy_(i32(p)); want.copy_(i32(w))
        graph.replay()
        torch.cuda.synchronize()
        ref = account(np.array(p), np.array(w), ref["held"], ref["table"], ref["free"], ref["n_free"][0], ps, n_pages, 64)
        same(dict(table=table.cpu().numpy(), held=held.cpu().numpy(), n_free=n_free.cpu().numpy(), flags=flags.cpu().numpy(),
                  start=start.cpu().numpy(), slots=slots.cpu().numpy()), ref)
