"""Log probabilities at an infinite temperature: all tokens that no mask excludes are alike, in every form that a row is taken in."""
import math

import pytest
import torch

from paper_2401_06706_amd import binding as M
from tests.test_gpu_chunk import DEV, gen
from tests.test_gpu_logprobs import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,V", [(3, 60), (3, 3000), (300, 517), (300, 9000), (300, 60001), (3, 120001)])
def test_infinite_temperature(rows, V, dtype):
    """One workgroup a row with 128 to 1024 threads, several a row; rows without a mask, with few tokens left, with one, and with values as low as the type has."""
    logits = (3 * torch.randn(4, V, generator=gen(V))).to(dtype)
    logits[1] = torch.where(torch.rand(V, generator=gen(1)) < 0.7, torch.tensor(-math.inf, dtype=dtype), logits[1])
    logits[1, 5], logits[1, 6] = 0.5, -math.inf
    logits[2] = -math.inf
    logits[2, V // 2] = 1.0
    logits[3, ::3] = torch.finfo(dtype).min
    n_top = 7
    which = [i % 4 for i in range(rows)] if rows > 4 else [0, 1, 2]
    tokens = [(5, 6, V // 2, 3)[r] for r in which]
    got = run(logits.to(DEV), tokens, n_top, [math.inf] * rows, which)
    for i, r in enumerate(which):
        z = logits[r].double()
        left = int((z > -math.inf).sum())
        want = -math.log(left)
        order = torch.sort(z, descending=True, stable=True).indices[:n_top].tolist()
        assert int(got["flags"][i]) == 0 and got["top_tok"][i].tolist() == order
        assert int(got["rank"][i]) == int(((z > z[tokens[i]]) | ((z == z[tokens[i]]) & (torch.arange(V) < tokens[i]))).sum())
        # Every weight is 1, so that their sum is exact: the logarithm's and the result's rounding.  The lowest values of a type are taken at 2^-149 of
        # them, which their weights and sums of V / 128 at most are rounded for.
        bound = 2.0 ** -24 * (2 + 2 * abs(want))
        if r == 3:
            bound += 2.0 ** -149 * 2.0 ** 128 + 2.0 ** -24 * (V / 128 + 8)
        for lp, token in [(got["logprob"][i], tokens[i])] + list(zip(got["top_logprob"][i], order)):
            assert float(lp) == -math.inf if z[token] == -math.inf else abs(float(lp) - want) <= bound, (i, token, float(lp), want)
        assert abs(float(got["entropy"][i]) + want) <= 2 * bound


def test_infinite_temperature_without_numbers():
    """What is no number is still refused."""
    logits = torch.randn(3, 100, generator=gen(2))
    logits[0, 3], logits[1, 4], logits[2] = float("nan"), math.inf, -math.inf
    got = run(logits.to(DEV), [1, 1, 1], 2, [math.inf] * 3)
    assert got["flags"].tolist() == [M.FLAG_NONFINITE] * 3 and torch.isnan(got["logprob"]).all() and torch.isnan(got["entropy"]).all()
