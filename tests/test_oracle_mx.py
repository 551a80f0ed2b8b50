"""Pins of the 4-bit oracle: hand-worked blocks, ties, the ends of the range, the blob's bytes (CPU)."""
import numpy as np
import pytest

from oracle import mx


def _values(v):
    return mx.values(np.array([v], np.float64))[0]


def test_every_member_of_a_block_with_scale_one_is_itself():
    v = np.concatenate([mx.MEMBERS, -mx.MEMBERS])
    codes, scales = mx.encode(v[None])
    assert scales.tolist() == [[127]] and codes[0].tolist() == list(range(16))
    assert np.array_equal(mx.decode(codes, scales)[0], v)


@pytest.mark.parametrize("x,want", [(0.25, 0.0), (0.2501, 0.5), (0.75, 1.0), (0.7499, 0.5), (1.25, 1.0), (1.75, 2.0), (2.5, 2.0), (3.5, 4.0),
                                    (3.4999, 3.0), (5.0, 4.0), (5.0001, 6.0), (6.999, 6.0), (7.999, 6.0)])
def test_ties_go_to_the_even_mantissa_and_what_is_past_six_to_six(x, want):
    got = _values([4.0, x, -x] + [0.0] * 29)
    assert got[1] == want and got[2] == -want


@pytest.mark.parametrize("a,s", [(4.0, 0), (7.99, 0), (8.0, 1), (3.99, -1), (2.0 ** -120, -122), (2.0 ** -125, -127), (2.0 ** -140, -127),
                                 (0.0, -127), (3.4e38, 125)])
def test_scale_of_the_largest_magnitude(a, s):
    assert mx.encode(np.array([[a, a / 2]]))[1][0, 0] == s + 127


def test_blocks_are_independent_and_the_last_may_be_short():
    x = np.zeros((2, 70))
    x[0, 0], x[0, 33], x[1, 69] = 1.0, 100.0, -0.01
    v = mx.values(x)
    assert v[0, 0] == 1.0 and v[0, 33] == 96.0 and abs(v[1, 69] + 0.01) <= 0.01 * 2 ** -2 and (v != 0).sum() == 3


def test_a_block_with_an_infinity_or_nan_is_nan_and_its_neighbours_are_not():
    x = np.ones((3, 96))
    x[1, 40], x[2, 0] = np.inf, np.nan
    v = mx.values(x)
    bad = np.isnan(v)
    assert bad[1, 32:64].all() and bad[2, :32].all() and bad.sum() == 64


def test_blob_bytes_of_a_small_matrix():
    x = np.zeros((33, 40))
    x[32, 1], x[0, 33] = 1.0, -3.0
    codes, scales = mx.encode(x)
    b = mx.blob(codes, scales)
    assert b.size == 128 + 512 + -(-33 * 32 // 128) * 128
    # row 32 lies in the second word of a 16-byte group; 1.0 is 4 times 2^-2 (code 6), column 1 is nibble 4
    assert b[128 + 0 * 16 + 1 * 4 + 0] == 125 and b[640 + 32 * 32 + 2] == 6
    # -3.0 is -6 times 2^-1 (code 15), column 33 of row 0 is nibble 4 of the fifth word
    assert b[128 + 1] == 126 and b[640 + 16 + 2] == 15
    assert (b[640:] != 0).sum() == 2


def test_product_of_values_equals_the_sum_over_blocks_of_scaled_integer_products():
    g = np.random.default_rng(5)
    x, w = g.normal(size=(3, 77)), g.normal(size=(4, 77))
    (cx, sx), (cw, sw) = mx.encode(x), mx.encode(w)
    ints = lambda c: (2 * mx.MEMBERS[c & 7]).astype(np.int64) * np.where(c & 8, -1, 1)
    y = np.zeros((3, 4))
    for b in range(3):
        part = ints(cx)[:, 32 * b:32 * b + 32] @ ints(cw)[:, 32 * b:32 * b + 32].T
        y += part * 0.25 * np.ldexp(1.0, sx[:, b].astype(int) - 127)[:, None] * np.ldexp(1.0, sw[:, b].astype(int) - 127)[None]
    assert np.allclose(y, mx.linear(mx.decode(cx, sx), mx.decode(cw, sw)), rtol=1e-13)
