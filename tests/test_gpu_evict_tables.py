"""Eviction with table entries outside the pool, in either table: rows that lie there, or were to go there, stay; their sequences are flagged; all else moves."""
import pytest
import torch

from paper_2401_06706_amd import binding as M
from tests import chunk_ref as R
from tests.test_gpu_chunk import DEV, gen

pytestmark = pytest.mark.gpu

PAGE, N_PAGES, H_KV, CAP = 32, 40, 2, 160
BAD = [-1, N_PAGES, 2 ** 31 - 1, -2 ** 31]


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.bfloat16, 40), (torch.float32, 64), (torch.float32, 256)])
@pytest.mark.parametrize("layers", [1, 3])
@pytest.mark.parametrize("fresh", [False, True])
def test_entries_outside_the_pool(fresh, layers, dtype, d):
    """Sequence 0: none.  1: in the middle of where rows come from.  2: where they go to.  3: where neither is.  4: everything kept, one page outside."""
    g = gen(91)
    lens, keeps = [150, 150, 140, 100, 60], [70, 66, 90, 40, 60]
    order = torch.randperm(N_PAGES, generator=g).int()
    table, other = order[:20].clone().view(4, 5), order[20:40].clone().view(4, 5)
    # (sequence 4 stands in pages that sequence 3 has no use for)
    table = torch.cat((table, torch.tensor([[int(table[3, 4])] + BAD], dtype=torch.int32)))
    other = torch.cat((other, torch.tensor([[int(other[3, 4]), int(other[3, 3])] + BAD[1:]], dtype=torch.int32)))
    table[1, 3], table[3, 4] = BAD[0], BAD[2]
    (other if fresh else table)[2, 1] = BAD[1]
    if fresh:
        other[3, 2], other[3, 3], other[3, 4] = BAD[3], BAD[0], BAD[1]
    k = torch.randn(layers, N_PAGES, H_KV, PAGE, d, generator=g).to(dtype)
    v = torch.randn(layers, N_PAGES, H_KV, PAGE, d, generator=g).to(dtype)
    sums = torch.rand(layers, 5, H_KV, CAP, generator=g)
    want = [k.clone(), v.clone()]
    kept_want, bad = {}, [False] * 5
    to = other if fresh else table
    inside = lambda p: 0 <= p < N_PAGES
    for l in range(layers):
        for b, n in enumerate(lens):
            for h in range(H_KV):
                pos = kept_want[l, b, h] = R.evicted(n, keeps[b], 2, 5, sums[l, b, h].tolist())
                for j, i in enumerate(pos):
                    src, dst = int(table[b, i // PAGE]), int(to[b, j // PAGE])
                    if not fresh and i == j:
                        continue                        # (a row that stays is not looked at)
                    if not (inside(src) and inside(dst)):
                        bad[b] = True
                        continue
                    for pool, w in ((k, want[0]), (v, want[1])):
                        w[l, dst, h, j % PAGE] = pool[l, src, h, i % PAGE]
    assert bad == [False, True, True, False, fresh]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    kd, vd, prefix, flags = k.to(DEV), v.to(DEV), i32(lens), i32([5] * 5)
    kept = torch.full((layers, 5, H_KV, CAP), -7, dtype=torch.int32, device=DEV)
    M.mcsd_kv_evict_paged(M.evict_args(kd, vd, table.to(DEV), sums.to(DEV), prefix, i32(keeps), kept, flags, 2, 5, other.to(DEV) if fresh else None))
    torch.cuda.synchronize()
    assert prefix.tolist() == keeps and flags.tolist() == [M.FLAG_BAD_PAGES if x else 0 for x in bad]
    for (l, b, h), pos in kept_want.items():
        assert kept[l, b, h, :len(pos)].tolist() == pos
    assert torch.equal(kd.cpu(), want[0]) and torch.equal(vd.cpu(), want[1])
