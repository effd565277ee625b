"""The oracle of a cache in 4 bits against numbers worked out by hand."""
import numpy as np
import pytest

from oracle import packed as P


def test_scales_are_the_upper_bits_of_fp16():
    for b in range(227):
        want = np.array([b << 7], np.uint16).view(np.float16)[0]
        assert P.scale_of(b) == float(want)
    assert P.scale_of(226) == 10240.0 and P.scale_of(255) == 10240.0 and P.scale_of(8) == 2.0 ** -14


def test_scale_is_the_nearest_of_a_sixth():
    assert P.scale_byte(6.0) == 15 << 3                       # 1
    assert P.scale_byte(0.0) == 8
    assert P.scale_byte(6 * 1.0625) == 15 << 3                # half-way to 1.125: the even one
    assert P.scale_byte(6 * 1.1875) == (15 << 3) + 2          # half-way from 1.125 to 1.25: the even one
    assert P.scale_byte(np.nextafter(6 * 1.0625, 9)) == (15 << 3) + 1
    assert P.scale_byte(6 * 1.9375) == 16 << 3                # half-way to the next power of two
    assert P.scale_byte(1e9) == 226 and P.scale_byte(3.4e38) == 226 and P.scale_byte(6e-6) == 8


@pytest.mark.parametrize("x, i", [(0, 0), (.25, 0), (.26, 1), (.74, 1), (.75, 2), (1.25, 2), (1.3, 3), (1.75, 4),
                                  (2.5, 4), (2.51, 5), (3.5, 6), (5, 6), (5.01, 7), (100, 7)])
def test_codes_are_nearest_with_ties_to_even(x, i):
    assert P.code_of(x * 0.75, 0.75) == i
    assert P.code_of(-x * 0.75, 0.75) == (i | 8 if x else i)
    assert P.code_of(-0.0, 1.0) == 8 and P.code_of(-3.4e38, 1.0) == 15


def test_rows_by_hand():
    x = np.zeros((1, 32))
    x[0, :4] = [6, -3, 0.5, 1]
    x[0, 16:19] = [-12, 4, np.nan]
    codes, scales = P.store(x)
    assert codes.shape == (1, 16) and scales.tolist() == [[120, 128, 0, 0]]
    assert codes[0, :2].tolist() == [7 | (8 | 5) << 4, 1 | 2 << 4]
    assert codes[0, 8:10].tolist() == [15 | 4 << 4, 0]
    got = P.values(codes, scales)
    assert got[0, :4].tolist() == [6, -3, 0.5, 1] and got[0, 16:19].tolist() == [-12, 4, 0]


def test_what_was_stored_is_stored_as_it_is():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((40, 48)) * np.exp(rng.uniform(-14, 13, (40, 1)))
    codes, scales = P.store(x)
    assert scales.shape == (40, 4) and P.store(np.zeros((2, 80)))[1].shape == (2, 8)
    again = P.store(P.values(codes, scales))
    assert (again[0] == codes).all() and (again[1] == scales).all()


def test_error_is_within_the_format():
    """Half a step of the grid: at most an eighth of the group's largest magnitude, give or take its clipping."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 16))
    err = np.abs(P.values(*P.store(x)) - x).max(1)
    assert (err <= np.abs(x).max(1) * (1 / 6) * 1.0625).all()
