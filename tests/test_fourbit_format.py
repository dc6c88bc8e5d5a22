"""The 4-bit form by itself, on the CPU: the test reference's two ways of encoding agree with each other, and values stay as near as the
header says."""
import numpy as np
import pytest

from tests import fourbit_ref as F


def blocks(seed):
    rng = np.random.default_rng(seed)
    yield np.zeros(32)
    yield np.full(32, -1.0)
    for e in (-130, -119, -20, 0, 60, 126):
        yield rng.normal(size=32).astype(np.float32) * 2.0 ** e
        yield np.concatenate((F.MAGNITUDES, -F.MAGNITUDES, (F.MAGNITUDES[1:] + F.MAGNITUDES[:-1]) / 2, [7.0, -6.5, 5.999, 0.2501, 0.2499, 0.74, 0.76, -2.5, 3.5])) * 2.0 ** e
    yield np.r_[np.ones(31), 7.0000001]
    yield np.r_[np.ones(31), np.nan]
    yield np.r_[np.ones(31), -np.inf]


@pytest.mark.parametrize("seed", range(3))
def test_both_encoders_agree_and_errors_are_within_the_documented(seed):
    for x in blocks(seed):
        code, s = F.encode_block(x)
        c2, s2 = F.encode(np.asarray(x)[None])
        assert s == s2[0, 0] and (code == c2[0, 0]).all()
        back = F.decode(c2, s2)[0]
        if s == 255:
            assert np.isnan(back).all()
            continue
        e = int(s) - 127
        assert -119 <= e <= 125
        if np.abs(x).max() <= 7.0 * 2.0 ** 125:
            assert (np.abs(back - x) <= np.maximum(np.abs(x) / 5, 2.0 ** e / 4) * (1 + 1e-12)).all()
            assert e == -119 or np.abs(x).max() > 3.5 * 2.0 ** e


def test_layout_of_a_pool():
    """One marked value per place: page, head, row and column come back where the header puts them."""
    P, H, ps, d = 2, 3, 64, 96
    codes = np.zeros((P, H, ps // 16, d // 32, 16, 16), np.uint8)
    scales = np.full((P, H, ps // 16, d // 32, 16), 127, np.uint8)
    flat = codes.reshape(-1)
    page, head, row, col = 1, 2, 37, 70
    block = ((((page * H + head) * (ps // 16) + row // 16) * (d // 32) + col // 32) * 16 + row % 16)
    flat[block * 16 + (col % 32) // 2] = 5 << (4 * (col % 2))
    rows = F.pool_rows(codes, scales)
    assert rows.shape == (P, H, ps, d) and rows[page, head, row, col] == 3.0 and (rows != 0).sum() == 1
