"""Attention over the 4-bit cache, few cut sequences among many: their partials are merged by all workgroups of the merge, whichever of the
sequences they are."""
import numpy as np
import pytest

from tests.fourbit_plan import plan_of, segments_of
from tests.test_gpu_fourbit import AttnCase, chain, random_tree

pytestmark = pytest.mark.gpu


def lengths(B, long, at, short):
    lens = [short - b % 7 for b in range(B)]
    for i, b in enumerate(at):
        lens[b] = long + 33 * i
    return lens


@pytest.mark.parametrize("B,H_q,H_kv,d,N,tree,at,long,short", [
    (70, 8, 8, 64, 28, random_tree, [3, 66, 69], 6000, 40),              # in both of the 64 sequences that are looked at together
    (130, 8, 4, 96, 3, chain, [0, 63, 64, 127, 128, 129], 9000, 30),
    (16, 32, 32, 128, 60, random_tree, [1, 4, 5, 9, 11, 15], 3000, 60),  # 1536 units of rows for 1024 workgroups
    (30, 8, 8, 256, 30, random_tree, [0, 7, 19], 4000, 60),
    (500, 2, 2, 32, 2, chain, [499], 20000, 20),
])
def test_few_cut_sequences(B, H_q, H_kv, d, N, tree, at, long, short):
    lens = lengths(B, long, at, short)
    c = AttnCase(B, H_q, H_kv, d, lens, N, tree, 64)
    plan = plan_of(c.args.desc)
    n = segments_of(c.args.desc, plan, lens)
    assert plan.bias == 0 and [b for b in range(B) if n[b] > 1] == at, n
    c.run()
    c.check(sorted({0, 1, B - 1, *at}))


def test_none_is_cut():
    lens = [300 + b for b in range(32)]
    c = AttnCase(32, 16, 16, 128, lens, 20, random_tree, 64, capacity=4000)
    plan = plan_of(c.args.desc)
    assert plan.n_segments_max > 1 and set(segments_of(c.args.desc, plan, lens)) == {1}
    c.run()
    c.check([0, 1, 31])
