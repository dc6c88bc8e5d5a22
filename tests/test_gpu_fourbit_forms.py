"""Attention over the 4-bit cache: every kernel that a launch can take, with sequences that stay whole and with sequences that are cut, against 64
bits.  What a case is meant to reach is checked on the host before it runs."""
import numpy as np
import pytest
import torch

from tests.fourbit_plan import form_of, plan_of, segments_of
from tests.test_gpu_fourbit import AttnCase, chain, i32, random_tree, star

pytestmark = pytest.mark.gpu

# rows per KV head: nodes, query heads per KV head, (tiles per wavefront, row groups) at d = 128 (below at most (2, 1), above (1, 1))
ROWS = [(1, 4, (1, 1)), (5, 3, (1, 1)), (7, 4, (2, 1)), (20, 3, (2, 2)), (33, 4, (2, 4))]


@pytest.mark.parametrize("cut", [False, True], ids=["whole", "cut"])
@pytest.mark.parametrize("rows", ROWS, ids=lambda r: f"{r[0]}x{r[1]}")
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 224, 256])
def test_every_form(d, rows, cut):
    N, G, small = rows
    lens = [4990, 1301] if cut else [190, 33]
    c = AttnCase(2, 2 * G, 2, d, lens, N, [chain, random_tree, star][d // 32 % 3], 32 if N < 7 else 96, root_row=N == 7, capacity=lens[0] + 90)
    plan = plan_of(c.args.desc)
    form = (1, 1) if d > 128 else small if d == 128 else min(small, (2, 1))
    assert form_of(c.args.desc, plan) == (64 if d <= 64 else 128 if d <= 128 else 256,) + form
    n = segments_of(c.args.desc, plan, lens)
    assert (min(n) > 1) if cut else (max(n) == 1), n
    c.run()
    c.check()
    # the same with entries that are no pages: the first, one in the middle, the last (which is not full)
    table, last = c.table, -(-lens[0] // c.ps) - 1
    table[0, 0], table[0, last // 2], table[0, last] = -1, c.n_pages, 2 ** 31 - 1
    c.cache.keep[4].copy_(i32(table))
    c.out.fill_(9.0)
    c.run()
    c.check()


def test_several_row_tiles():
    for d, N, G, groups in ((64, 40, 3, 1), (96, 25, 4, 1), (128, 60, 3, 4), (256, 50, 2, 1)):
        for lens in ([300, 0], [3000, 2000]):
            c = AttnCase(2, 2 * G, 2, d, lens, N, random_tree, 64)
            plan = plan_of(c.args.desc)
            assert plan.n_row_tiles > 1 and form_of(c.args.desc, plan)[2] == groups
            assert (max(segments_of(c.args.desc, plan, lens)) > 1) == (lens[0] == 3000)
            c.run()
            c.check()


def test_short_sequences_have_the_same_bits_whatever_capacity_is_named():
    a = AttnCase(2, 8, 2, 64, [90, 33], 10, random_tree, 32, capacity=96)
    b = AttnCase(2, 8, 2, 64, [90, 33], 10, random_tree, 32, capacity=30000)
    for c in (a, b):
        assert segments_of(c.args.desc, plan_of(c.args.desc), c.lens) == [1, 1]
        c.run()
    torch.cuda.synchronize()
    assert torch.equal(a.q, b.q) and torch.equal(a.out.view(torch.int16), b.out.view(torch.int16))
    a.check()
