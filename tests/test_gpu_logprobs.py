"""Log probabilities of given tokens on the GPU: values against 64 bits, ranks and ids to the bit."""
import math

import pytest
import torch

from paper_2401_06706_amd import binding as M
from tests import chunk_ref as R
from tests.test_gpu_chunk import DEV, gen

pytestmark = pytest.mark.gpu


def run(logits, tokens, n_top, temperature=None, row_map=None):
    rows = len(tokens)
    i32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)
    f = lambda *s: torch.full(s, 9.0, device=DEV)
    i = lambda *s: torch.full(s, 9, dtype=torch.int32, device=DEV)
    o = {"logprob": f(rows), "entropy": f(rows), "rank": i(rows), "flags": i(rows), "top_tok": i(rows, n_top) if n_top else None,
         "top_logprob": f(rows, n_top) if n_top else None}
    toks = i32(tokens)
    need = M.mcsd_logprob_workspace_bytes(M.logprob_desc(logits, toks, n_top))
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device=DEV) if need else None
    t = None if temperature is None else torch.tensor(temperature, dtype=torch.float32, device=DEV)
    M.mcsd_token_logprobs(M.logprob_args(logits, toks, o["logprob"], o["entropy"], o["rank"], o["top_tok"], o["top_logprob"], o["flags"], t, i32(row_map), ws))
    torch.cuda.synchronize()
    return {k: None if v is None else v.cpu() for k, v in o.items()}


def check(logits, tokens, n_top, temperature=None, row_map=None):
    got = run(logits, tokens, n_top, temperature, row_map)
    host, V = logits.cpu(), logits.shape[1]
    for i, x in enumerate(tokens):
        T = 1.0 if temperature is None else float(torch.tensor(temperature[i], dtype=torch.float32))
        r = i if row_map is None else row_map[i]
        want = R.logprobs(host[r], x, T, n_top) if 0 <= r < logits.shape[0] else None
        if want is None:
            assert int(got["flags"][i]) == (M.FLAG_NONFINITE if 0 <= r < logits.shape[0] else M.FLAG_BAD_TREE)
            assert math.isnan(got["logprob"][i]) and math.isnan(got["entropy"][i]) and int(got["rank"][i]) == -1
            assert n_top == 0 or ((got["top_tok"][i] == -1).all() and torch.isnan(got["top_logprob"][i]).all())
            continue
        lp, entropy, rank, ids, tops = want
        T = T if T > 0 else 1.0
        z = host[r].double()
        spread = float((z.max() - z[x]) / T) if 0 <= x < V and z[x] > -math.inf else 0.0
        assert int(got["flags"][i]) == (0 if 0 <= x < V else M.FLAG_BAD_TOKEN)
        assert int(got["rank"][i]) == rank
        if n_top:
            assert got["top_tok"][i].tolist() == ids
        def near(a, b, s):
            return a == b or (math.isnan(a) and math.isnan(b)) or abs(a - b) <= R.logprob_bound(V, b, s)
        assert near(float(got["logprob"][i]), lp, spread), (float(got["logprob"][i]), lp)
        for a, b in zip(got["top_logprob"][i].tolist() if n_top else [], tops):
            assert near(a, b, float(abs(b)) + entropy if b > -math.inf else 0.0), (a, b)
        # lse and a mean of (z - max) / T, each off by as much of itself
        assert abs(float(got["entropy"][i]) - entropy) <= 2 * R.logprob_bound(V, entropy, entropy) * (1 + entropy), (float(got["entropy"][i]), entropy)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 7, 64, 100, 511, 1000, 4099, 32000, 50001, 151936, 262144])
def test_rows(V, dtype):
    logits = (3 * torch.randn(5, V, generator=gen(V))).to(dtype).to(DEV)
    tokens = [0, V - 1, V // 2, int(logits[3].argmax()), int(logits[4].argmin())]
    for n in {0, 1, min(V, 5), min(V, 20), min(V, 64)}:
        check(logits, tokens, n, [1.0, 0.0, 0.3, 2.0, 0.7])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [70, 3001, 40000])
def test_ties_and_masks(V, dtype):
    rows = [torch.zeros(V), torch.full((V,), -math.inf), torch.randint(0, 3, (V,), generator=gen(1)).float(), torch.full((V,), torch.finfo(dtype).min),
            torch.arange(V).float().neg().div(64).floor(), torch.randn(V, generator=gen(2)), torch.randn(V, generator=gen(3)), torch.randn(V, generator=gen(4)),
            torch.randn(V, generator=gen(5)), torch.randn(V, generator=gen(6))]
    rows[1][V // 3] = 2.0
    rows[5][:] = torch.where(torch.rand(V, generator=gen(7)) < 0.9, torch.tensor(-math.inf), rows[5])
    rows[5][3] = 0.5
    rows[6][5:] = -math.inf
    rows[7][V - 6:] = rows[7].max() + 1
    rows[8][::2], rows[8][1] = -0.0, 0.0
    rows[9][V // 2] = torch.finfo(dtype).max / 2
    logits = torch.stack(rows).to(dtype).to(DEV)
    for n in {1, 20, 64}:
        check(logits, [V // 3, V // 3, 2, 1, V - 1, 3, 4, V - 1, 0, 5], n)
        check(logits, [0] * 10, n)


def test_more_above_the_bound_than_fit():
    """All large logits in the pieces of few threads: the top is then looked for one by one."""
    V = 512 * 4 * 300
    row = torch.randn(V, generator=gen(1))
    own = (torch.arange(V) // 4) % 512
    row[own < 3] += 100.0                               # 3600 logits of three threads
    logits = torch.stack((row, row.flip(0))).to(DEV)
    for n in (1, 3, 4, 5, 64):
        check(logits, [0, 17], n)
    for n in (5, 64):
        check(logits.bfloat16(), [0, 17], n)


def test_no_numbers_and_bad_rows():
    V = 5000
    logits = torch.randn(4, V, generator=gen(1))
    logits[0, 77], logits[1, 4999], logits[2] = float("nan"), float("inf"), -float("inf")
    check(logits.to(DEV), [0, 1, 2, 3], 4)
    check(logits.to(DEV), [5, 6, 7, 8, V, -1], 4, row_map=[3, -1, 4, 3, 3, 3])
    check(logits.to(DEV), [2, V + 5], 0, row_map=[3, 3])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", range(0, 9))
def test_rows_that_start_anywhere(shift, dtype):
    """Row strides and starts of any alignment; a row is read no farther than its V logits."""
    V, stride = 517, 523 + shift
    flat = torch.full((4 * stride + shift + 16,), float("nan"), dtype=dtype)
    view = flat[shift:shift + 4 * stride].view(4, stride)[:, :V]
    view.copy_(torch.randn(4, V, generator=gen(shift)))
    flat = flat.to(DEV)
    logits = flat[shift:shift + 4 * stride].view(4, stride)[:, :V]
    check(logits, [0, 516, 8, 300], 20)


def test_no_rows():
    run(torch.randn(3, 100, device=DEV), [], 5)
    run(torch.randn(3, 100, device=DEV), [], 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,V,n_top", [(257, 515, 3), (300, 2500, 20), (700, 33, 40), (2000, 1, 1)])
def test_more_rows_than_workgroups(rows, V, n_top, dtype):
    """Where a row is shared by half as many threads, with row_map backwards, one row named twice and some beyond the last."""
    logits = (3 * torch.randn(rows, V + 5, generator=gen(rows))).to(dtype).to(DEV)[:, :V]
    row_map = [rows - 1 - i for i in range(rows)]
    row_map[7], row_map[8], row_map[9] = row_map[6], rows, -1
    tokens = torch.randint(0, V, (rows,), generator=gen(V)).tolist()
    check(logits, tokens, min(n_top, V), [0.5 + (i % 5) / 2 for i in range(rows)], row_map)


@pytest.mark.parametrize("rows,V,dtype", [(3, 2048, torch.bfloat16), (3, 2049, torch.bfloat16), (3, 1025, torch.float32), (260, 8192, torch.float32),
                                          (260, 8193, torch.float32), (260, 57344, torch.bfloat16), (260, 57345, torch.bfloat16), (260, 28673, torch.float32)])
def test_threads_of_a_row(rows, V, dtype):
    """Around the sizes where a row is taken by more threads."""
    logits = (3 * torch.randn(rows, V, generator=gen(V))).to(dtype).to(DEV)
    ids = list(range(0, rows, max(1, rows // 9)))
    check(logits, [(7919 * i) % V for i in range(len(ids))] + [0] * 250, 20, row_map=ids + [ids[1]] * 250) if rows > 256 else check(logits, [0, V - 1, V // 2], 20)


def test_temperatures_at_the_ends():
    """The smallest numbers leave the largest logit alone, the largest make all logits equal; 0 reads as 1."""
    logits = torch.randn(5, 300, generator=gen(3)).to(DEV)
    best = logits.argmax(1).tolist()
    got = run(logits, best, 2, [1e-45, 1e-38, 3e38, 0.0, 1.0], [0, 1, 2, 3, 3])
    assert got["flags"].tolist() == [0] * 5 and got["rank"].tolist()[:4] == [0] * 4
    for i in (0, 1):
        assert float(got["logprob"][i]) == 0.0 and float(got["entropy"][i]) == 0.0
        assert int(got["top_tok"][i, 0]) == best[i] and float(got["top_logprob"][i, 0]) == 0.0 and float(got["top_logprob"][i, 1]) < -1e30
    bound = R.logprob_bound(300, math.log(300), 0)
    assert abs(float(got["logprob"][2]) + math.log(300)) <= bound and abs(float(got["entropy"][2]) - math.log(300)) <= 2 * bound * (1 + math.log(300))
    for k in ("entropy", "top_logprob"):
        assert torch.equal(got[k][3], got[k][4])


@pytest.mark.parametrize("V,dtype,shift", [(52001, torch.float32, 0), (60001, torch.float32, 3), (110003, torch.bfloat16, 5), (262144, torch.float32, 0)])
def test_rows_in_parts(V, dtype, shift):
    """Long rows that several workgroups share: ties across their borders, parts that a mask leaves empty or nearly so, tokens of every part, rows that start
    anywhere, what is no number in one part alone."""
    inf = math.inf
    rows = [torch.randn(V, generator=gen(1)), torch.zeros(V), torch.full((V,), -inf), torch.randint(0, 3, (V,), generator=gen(2)).float(),
            torch.full((V,), torch.finfo(dtype).min), torch.full((V,), -inf), torch.full((V,), -inf), torch.full((V,), -inf), torch.randn(V, generator=gen(3)),
            torch.randn(V, generator=gen(4)), torch.full((V,), -inf), torch.where(torch.rand(V, generator=gen(5)) < 0.001, torch.randn(V, generator=gen(6)), torch.tensor(-inf))]
    rows[2][V // 2] = 1.0                               # one token
    rows[5][:30] = torch.randn(30, generator=gen(7))    # the first part alone
    rows[6][V - 30:] = 0.5                              # the last
    rows[7][::V // 25] = 2.0                            # a few of each, all alike
    rows[8][V - 3], rows[9][V // 3] = float("nan"), inf
    flat = torch.full((len(rows) * (V + 7) + shift,), float("nan"))
    view = flat[shift:].view(len(rows), V + 7)[:, :V]
    view.copy_(torch.stack(rows))
    flat = flat.to(dtype).to(DEV)
    logits = flat[shift:].view(len(rows), V + 7)[:, :V]
    for n_top in (0, 1, 20, 64):
        check(logits, [0, V - 1, V // 2, V // 3, 7, 29, V - 1, V // 25, 5, 5, 5, V // 2], n_top)
    check(logits, [(V * i) // 9 for i in range(9)] + [V, -1, 3, 3], 5, [0.3 + i / 4 for i in range(13)], [0] * 11 + [len(rows), -1])
