"""Pages from lengths at the borders of the kernels that a call can take: 64, 256 and 1024 threads, a slot map in the same launch or in its own,
more sequences than threads; against the sequential account."""
import numpy as np
import pytest

from tests.test_gpu_pages import account, run, same, state

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("wanted", ["fits", "ends early"])
@pytest.mark.parametrize("B,max_slots", [(64, 256), (64, 257), (65, 256), (256, 257), (256, 2048), (256, 2049), (257, 1), (257, 2048), (257, 2049), (512, 1500),
                                         (700, 2048), (1023, 900), (1024, 2048), (1024, 2049), (1025, 2048), (1025, 2049)])
def test_at_the_borders(B, max_slots, wanted):
    rng = np.random.default_rng(B + max_slots)
    ps, most, spare = 32, 300, B // 2
    prefix, held, table, free, n_pages = state(rng, B, ps, most, spare)
    new = max(1, max_slots // (2 * B)) if wanted == "fits" else 3 * max_slots // B + 3
    want = np.minimum(prefix + rng.integers(0, new + 1, size=B), table.shape[1] * ps)
    want[rng.random(B) < 0.1] = 0
    want[rng.random(B) < 0.02] = table.shape[1] * ps + 1          # does not fit its table
    want[:3], want[-1] = prefix[:3], prefix[-1] + 1               # sequences without a slot first, one with a slot last
    prefix[7], want[B // 2], held[B - 3] = -1, -2, table.shape[1] + 1
    expect = account(prefix, want, held, table, free, spare, ps, n_pages, max_slots)
    assert (expect["flags"] & 512 > 0).sum() == 3
    if wanted == "ends early" and max_slots > 1:
        assert (expect["flags"] & 1024).any() and (expect["slots"] >= 0).any()
    got, _, _ = run(prefix, want, held, table, free, spare, ps, max_slots)
    same(got, expect)


@pytest.mark.parametrize("B", [1, 64, 65, 256, 257, 1024, 1025])
def test_without_a_slot_map(B):
    rng = np.random.default_rng(B)
    prefix, held, table, free, n_pages = state(rng, B, 64, 500, B)
    want = rng.integers(0, 900, size=B)
    got, _, _ = run(prefix, want, held, table, free, B, 64, 0, maps=False)
    same(got, account(prefix, want, held, table, free, B, 64, n_pages, 10 ** 6))       # (no map, none that could end too early)
