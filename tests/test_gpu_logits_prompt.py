"""Rules on logits where the prompt is as long as the history, longer (a window of the history was passed, or its length does not fit) or negative:
candidates are generated tokens all the same, so that they count."""
import numpy as np
import pytest
import torch

from paper_2401_06706_amd import binding as M
from tests.test_gpu_logits_rules import check, i32, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,inplace", [("fp32", False), ("fp32", True), ("bf16", False)])
def test_prompts_of_any_length(dtype, inplace):
    c = make(8, 2100, 9, 300, dtype=dtype, n_bias=3, allow=0.8)
    c["hist_len"] = np.array([300, 0, 300, 7, 7, 1000, -4, 299], np.int32)             # (taken within 0 .. 300)
    c["prompt_len"] = np.array([300, 5, 301, 2 ** 31 - 1, -3, 900, 2, -(2 ** 31)], np.int32)
    check(c, inplace)


def test_a_candidate_counts_whatever_the_prompt_is():
    V, tokens = 64, [5, 5, 9]
    z = torch.zeros(2, 2, V, device="cuda:0")
    f32 = lambda *v: torch.tensor(v, device="cuda:0")
    M.mcsd_logits_rules(M.logits_args(z, z, i32([-1]), i32([[5], [7]]), i32([tokens, tokens]), i32([3, 3]), i32([3, 40]),
                                      presence=f32(0.5, 0.5), frequency=f32(0.25, 0.25)))
    want = torch.zeros(2, 2, V)
    want[0, 1, 5] = want[1, 1, 7] = -0.75                     # the candidate alone; what the prompt holds is only seen
    assert torch.equal(z.cpu(), want)
