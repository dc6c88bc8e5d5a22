"""How exact the sums of the log probabilities are, form by form: bounds that follow the number of logits which one lane adds up."""
import math

import pytest
import torch

from tests import chunk_ref as R
from tests.test_gpu_chunk import DEV, gen
from tests.test_gpu_logprobs import run

pytestmark = pytest.mark.gpu
U = 2.0 ** -24

FORMS = [  # rows, V, dtype, lanes that share a row
    (4, 1000, torch.float32, 128), (4, 32000, torch.float32, 1024), (4, 50001, torch.bfloat16, 1024), (300, 8000, torch.float32, 128), (300, 16000, torch.bfloat16, 128),
    (300, 28000, torch.float32, 256), (300, 50001, torch.bfloat16, 256), (300, 32000, torch.float32, 512), (4, 151936, torch.float32, 512 * 12), (4, 262144, torch.float32, 512 * 16),
    (4, 262144, torch.bfloat16, 512 * 10),
]


@pytest.mark.parametrize("kind", ["normal", "flat", "rising"])
@pytest.mark.parametrize("rows,V,dtype,lanes", FORMS)
def test_bits(rows, V, dtype, lanes, kind):
    z = {"normal": lambda: 3 * torch.randn(4, V, generator=gen(V)), "flat": lambda: 0.01 * torch.randn(4, V, generator=gen(V)),
         "rising": lambda: torch.linspace(-12, 3, V).repeat(4, 1) + 0.1 * torch.randn(4, V, generator=gen(V))}[kind]().to(dtype)
    T = [1.0, 0.7, 1.3, 2.0]
    which = [i % 4 for i in range(rows)]
    tokens = [(7919 * i) % V for i in range(rows)]
    got = run(z.to(DEV), tokens, 3, [T[r] for r in which], which)
    for i in range(0, rows, max(1, rows // 12)):
        r = which[i]
        lp, entropy, rank, ids, tops = R.logprobs(z[r], tokens[i], T[r], 3)
        zd = z[r].double() / float(torch.tensor(T[r]))
        p = torch.softmax(zd, 0)
        t = zd.max() - zd
        mean, square = float((p * t).sum()), float((p * t * t).sum())
        n = V / lanes + 16                              # logits of a lane, those outside whole pieces among them
        # A weight 2^((z - m) c): log2(e), the quotient by T, the difference and the product are rounded, 4 U of the exponent, so 4 U t of the weight, and again
        # 4 U t over all rises of the maximum together; the exponential is off by a unit, 2 U.  A lane's sum takes n additions, and once per 16 logits
        # at most a factor: 3 U with its exponential.
        s = U * (8 * mean + 2 + n + 3 * (n / 16 + 8))
        for a, b, token in [(got["logprob"][i], lp, tokens[i])] + [(a, b, k) for a, b, k in zip(got["top_logprob"][i], tops, ids)]:
            # lse as its sum, (z - m) / T by the rounding of log2(e) / T, the result's own
            assert abs(float(a) - b) <= s + U * (3 * float(t[token]) + abs(b)), (float(a), b, s)
        # lse + sum p t: the weighted sum has each term's weight off as above, t itself by 4 U of it, products, additions and factors as before
        bound = s + U * (8 * square + (4 + 2 + 2 + n + 4 * (n / 16 + 8)) * mean) + s * mean + U * entropy
        assert abs(float(got["entropy"][i]) - entropy) <= bound, (float(got["entropy"][i]), entropy, bound)
