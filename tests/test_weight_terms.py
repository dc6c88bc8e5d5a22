"""How far off two bf16 terms leave a softmax weight, over all fp32 values of a binade: the first cut (one step lower where that is exact), as attention
over caches of full precision takes it, and the first rounded to nearest, as attention over the 4-bit cache does."""
import numpy as np

P = np.arange(0x3f800000, 0x40000000, dtype=np.uint32)


def nearest_bf16(x):
    u = x.astype(np.float32).view(np.uint32).astype(np.uint64)
    return ((u + ((u >> 16) & 1) + 0x7fff) & 0xffff0000).astype(np.uint32).view(np.float32).astype(np.float64)


def worst(hi):
    p = P.view(np.float32).astype(np.float64)
    return (np.abs(hi + nearest_bf16(p - hi) - p) / p).max()


def test_first_term_cut():
    assert 2.0 ** -17 < worst(((P - 1) & 0xffff0000).astype(np.uint32).view(np.float32).astype(np.float64)) <= 2.0 ** -16


def test_first_term_nearest():
    assert worst(nearest_bf16(P.view(np.float32))) <= 2.0 ** -17
