"""Long sequences with few rows: sixteen segments of keys and more, which the merge joins by groups of 32 lanes, at every padded head dimension."""
import math

import pytest
import torch

from tests import chunk_ref as R
from tests.test_gpu_chunk import DEV, check, gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,news,H_q,H_kv", [([16000], [1], 4, 2), ([9001], [13], 7, 1), ([5000, 12000, 3], [1, 3, 1], 6, 3)])
@pytest.mark.parametrize("d", [8, 32, 64, 80, 96, 112, 128, 136, 256])
def test_many_segments(d, lens, news, H_q, H_kv, dtype):
    """(segments of eight tiles of 32 keys: 63 of the first batch, 36 of the second, 20 and 47 of the third)"""
    check(R.make_batch(gen(81), DEV, dtype, lens, news, H_q, H_kv, d, 32), 1 / math.sqrt(d), dtype)
