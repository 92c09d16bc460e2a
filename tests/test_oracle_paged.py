"""The 4-bit blocks' oracle against hand-worked blocks and its own definition."""
import numpy as np
import pytest

from oracle import paged


def test_codes_by_hand():
    x = np.zeros(32)
    # largest 6 -> floor(log2) 2, exponent 0: the numbers themselves; ties go to the even code
    x[:16] = [6, -6, 0.25, 0.26, 0.74, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 5.01, -0.25, -1.25, 4.99, -5]
    codes, scale = paged.encode_block(x, "fp16")
    assert scale == 127
    assert codes[:16] == [7, 15, 0, 1, 1, 2, 2, 4, 4, 6, 6, 7, 8, 10, 6, 14] and codes[16:] == [0] * 16
    codes, scale = paged.encode_block(np.array([7.99] + [1.0] * 31), "fp16")   # beyond 6: 6
    assert scale == 127 and codes[0] == 7 and codes[1] == 2
    codes, scale = paged.encode_block(np.array([8.0, 1.0] + [0.0] * 30), "fp16")
    assert scale == 128 and codes[:3] == [6, 1, 0]


@pytest.mark.parametrize("dtype,smallest", [("fp16", 2.0 ** -24), ("bf16", 2.0 ** -133)])
def test_lowest_exponent_and_zeros(dtype, smallest):
    codes, scale = paged.encode_block(np.zeros(32), dtype)
    assert codes == [0] * 32 and scale == paged.LOWEST[dtype] + 127
    codes, scale = paged.encode_block(np.array([smallest] + [0.0] * 31), dtype)
    assert scale == paged.LOWEST[dtype] + 127 and codes[0] == (1 if dtype == "fp16" else 0)


def test_non_finite_blocks():
    for bad in (np.inf, -np.inf, np.nan):
        x = np.ones(128)
        x[40] = bad
        codes, scales = paged.encode_row(x, "bf16")
        assert list(scales) == [125, 255, 125, 125]
        back = paged.decode_rows(codes, scales)
        assert np.isnan(back[32:64]).all() and (back[:32] == 1).all() and (back[64:] == 1).all()


def test_round_trip_is_exact_on_the_grid_and_near_elsewhere():
    rng = np.random.default_rng(0)
    x = rng.standard_normal(128).astype(np.float16).astype(np.float64)
    back = paged.decode_rows(*paged.encode_row(x, "fp16"))
    again = paged.decode_rows(*paged.encode_row(back, "fp16"))
    assert np.array_equal(back, again)
    top = np.abs(x.reshape(4, 32)).max(1).repeat(32)
    # half of the largest step, 2 of 4 to 8 times 2^e; beyond 6 up to 2 2^e
    assert (np.abs(back - x) <= 2.0 ** (np.floor(np.log2(top)) - 2) * np.where(np.abs(x) > 6 * 2.0 ** (np.floor(np.log2(top)) - 2), 2, 1)).all()


def test_slots():
    assert list(paged.sequence_slots([5, 2, 9], 35, 16)) == [*range(80, 96), *range(32, 48), 144, 145, 146]
    pages = np.arange(3 * 2 * 16 * 128, dtype=np.float64).reshape(3, 2, 16, 128)
    r = paged.rows_of(pages, 16, [17, -1, 47, 48])
    assert np.array_equal(r[0], pages[1, :, 1]) and not r[1].any() and np.array_equal(r[2], pages[2, :, 15]) and not r[3].any()
