"""The 4-bit oracle, pinned by values worked out by hand, and the library's row size."""
import numpy as np
import pytest

import paper_2502_01637_amd as S
from oracle import mx4


def test_row_bytes():
    for cols, want in [(1, 80), (128, 80), (129, 144), (512, 272), (1000, 544), (1024, 544),
                       (2048, 1088), (1 << 22, 17 << 17)]:
        assert mx4.row_bytes(cols) == want == S.mx4_row_bytes(cols)
    for cols in (0, -5, (1 << 22) + 1):
        with pytest.raises(ValueError):
            S.mx4_row_bytes(cols)


def test_a_block_by_hand():
    x = np.zeros((1, 34))
    x[0, :12] = [6, -6, 4, 5, 7, 7.99, 0.25, 0.75, 2.5, 3.5, -0.1, 0.26]
    x[0, 33] = -3.0e-3
    r = mx4.quantize(x)
    assert r.shape == (1, 80)
    codes = np.stack([r[0, :64] & 15, r[0, :64] >> 4], 1).reshape(-1)
    # the block's largest magnitude lies in [4, 8): scale 1; ties go to even codes
    assert codes[:12].tolist() == [7, 15, 6, 6, 7, 7, 0, 2, 4, 6, 8, 1]
    assert r[0, 64] == 127
    # 3e-3 = 1.536 * 2^-9: scale 2^-11, 6.144 steps, 6 of them
    assert r[0, 65] == 127 - 11 and codes[33] == 15 and codes[32] == 0
    assert (r[0, 66:] == 0).all() and (codes[34:] == 0).all()
    v = mx4.values(r, 34)
    assert v[0, :12].tolist() == [6, -6, 4, 4, 6, 6, 0, 1, 2, 4, -0.0, 0.5]
    assert v[0, 33] == -6 * 2.0 ** -11


def test_edges_of_the_scale():
    tiny = np.float64(2.0) ** -149
    for x, s, v in [(0.0, 0, 0.0), (tiny, 0, 0.0), (2.0 ** -128, 0, 2.0 ** -128),
                    (2.0 ** -125, 0, 2.0 ** -125), (2.0 ** -124, 1, 2.0 ** -124),
                    (2.0 ** 127, 252, 2.0 ** 127), (np.float32(3.4028235e38), 252, 1.5 * 2.0 ** 127)]:
        r = mx4.quantize(np.array([[x]]))
        assert r[0, 64] == s and mx4.values(r, 1)[0, 0] == v
    for x in (np.inf, -np.inf, np.nan):
        r = mx4.quantize(np.array([[1.0, x] + [2.0] * 40]))
        assert r[0, 64] == 255 and (r[0, :16] == 0).all() and r[0, 65] == 126
        v = mx4.values(r, 42)
        assert np.isnan(v[0, :32]).all() and (v[0, 32:] == 2.0).all()


def test_the_vectorised_rounding_is_the_packed_one():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((9, 96)) * np.exp2(rng.integers(-20, 20, (9, 1)))
    x[3] = 0.0
    x[4, :9] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -7.5]
    assert np.array_equal(mx4.rounded(x), mx4.values(mx4.quantize(x), 96))
