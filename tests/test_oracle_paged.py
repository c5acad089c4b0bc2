"""Pins of the paged-cache oracle: E4M3 rounding and scales by hand and against torch's cast, pages."""
import numpy as np
import pytest
import torch

from oracle import block_attention
from oracle import paged


def test_e4m3_values():
    v = paged.e4m3_values()
    assert v[0x7E] == 448.0 and v[0x78] == 256.0 and v[0x38] == 1.0 and v[0x08] == 2.0 ** -6
    assert v[0x01] == 2.0 ** -9 and v[0x07] == 7 * 2.0 ** -9 and v[0xB8] == -1.0
    assert np.isnan(v[0x7F]) and np.isnan(v[0xFF]) and np.signbit(v[0x80])
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(v, t)


@pytest.mark.parametrize("y,code", [
    (0.0, 0x00), (-0.0, 0x80), (448.0, 0x7E), (-448.0, 0xFE), (432.0, 0x7E), (431.9, 0x7D),
    (1.0625, 0x38), (1.1875, 0x3A), (1.0626, 0x39), (2.0 ** -10, 0x00), (1.5 * 2.0 ** -9, 0x02),
    (2.0 ** -10 * 1.001, 0x01), (np.nan, 0x7F), (np.inf, 0x7F), (-np.inf, 0x7F)])
def test_rounding_by_hand(y, code):
    # 432 lies half way between 416 (0x7d, odd) and 448; 1.0625 between 1 (0x38) and 1.125
    assert paged.round_e4m3(np.array([y]))[0] == code


def test_rounding_against_the_cast():
    x = np.random.default_rng(0).standard_normal(20000) * np.exp(
        np.random.default_rng(1).uniform(-9, 4, 20000))
    x = np.clip(x, -448, 448).astype(np.float32)
    mid = (paged.e4m3_values()[:126] + paged.e4m3_values()[1:127]) / 2    # all ties
    x = np.concatenate([x, mid.astype(np.float32), -mid.astype(np.float32)])
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(paged.round_e4m3(x), want)


@pytest.mark.parametrize("a,e", [
    (448.0, 0), (448.0001, 1), (224.0, -1), (1.0, -8), (1.75, -8), (1.7501, -7), (0.0, -100),
    (448.0 * 2.0 ** -100, -100), (1e-38, -100), (3.4e38, 120), (448.0 * 2.0 ** 119, 119)])
def test_scale_by_hand(a, e):
    codes, s = paged.quantise(np.array([[a, -a / 2, 0.0]]))
    assert int(s[0]) - 127 == e
    if a >= 448.0 * 2.0 ** -100:
        # a 2^-e lies in (224, 448] and may round to 224 (1.7501 * 2^7 = 224.01)
        assert 224 <= paged.e4m3_values()[codes[0, 0]] <= 448


def test_values_off_by_at_most_half_a_step():
    x = np.random.default_rng(2).standard_normal((500, 64)) * np.exp(
        np.random.default_rng(3).uniform(-60, 60, (500, 1)))
    codes, s = paged.quantise(x)
    back = paged.dequantise(codes, s)
    least = 2.0 ** -10 * 2.0 ** (s.astype(float) - 127)[:, None]
    assert (np.abs(back - x) <= np.maximum(2.0 ** -4 * np.abs(x), least)).all()


def test_nonfinite_values_do_not_set_the_scale():
    codes, s = paged.quantise(np.array([[np.inf, 1.0, np.nan, -2.0]]))
    assert int(s[0]) - 127 == -7       # of 2.0: 448 * 2^-8 = 1.75 < 2
    np.testing.assert_array_equal(np.isnan(paged.dequantise(codes, s)), [[True, False, True, False]])


def test_pages():
    """Rows come back from where they were written; rows without a page are dropped or zero."""
    table = np.array([[3, 0, -1], [1, 9, 2]])
    pool = np.full((4, 2, 16, 4), np.nan)
    rng = np.random.default_rng(4)
    rows = rng.standard_normal((30, 2, 4))
    paged.kv_write(pool, table, rows, [0, 20, 30], [14, 5])
    back = paged.kv_read(pool, table, [34, 18])
    np.testing.assert_array_equal(back[14:32], rows[:18])         # positions 14 .. 31
    np.testing.assert_array_equal(back[32:34], 0)                 # no page
    np.testing.assert_array_equal(back[34 + 5:34 + 15], rows[20:])
    np.testing.assert_array_equal(back[-2:], 0)                   # page 9 of 4
    assert np.isnan(back[:14]).all()
    pos = [0, -1, 33, 40] + [-1] * 26
    paged.kv_write(pool, table, rows, [0, 20, 30], [14, 5], pos)  # 33: no page; 40: past the table
    np.testing.assert_array_equal(pool[3, :, 0], rows[0])


def test_attention_over_pages_is_attention_over_the_packed_prefix():
    rng = np.random.default_rng(5)
    table = np.array([[2, 0], [1, -1]])
    k, v = rng.standard_normal((2, 3, 2, 16, 8))
    q = rng.standard_normal((5, 4, 8))
    kb, vb = rng.standard_normal((2, 5, 2, 8))
    got = paged.paged_attention(q, kb, vb, k, v, table, [0, 2, 5], [19, 3], 4, 2)
    pre = [np.concatenate([np.concatenate([x[2].transpose(1, 0, 2), x[0].transpose(1, 0, 2)])[:19],
                           x[1].transpose(1, 0, 2)[:3]]) for x in (k, v)]
    np.testing.assert_array_equal(got, block_attention(q, kb, vb, *pre, [0, 2, 5], [0, 19, 22], 4, 2))
