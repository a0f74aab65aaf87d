"""The tests' own form of the codes: fields and roundings by hand."""
import numpy as np
import pytest

from codes_ref import bf16_bits, decode, encode, values


def test_values():
    v = values(8)
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[0x38] == 1 and v[0x39] == 1.125 and v[126] == 448
    assert (np.diff(v) > 0).all() and (np.diff(values(4)) > 0).all()


@pytest.mark.parametrize("bits,x,byte,code", [(8, 448.0, 127, 0x7E), (8, 452.0, 128, 0x76), (8, 1.75, 119, 0x7E), (8, 1.765625, 120, 0x76),
                                              (4, 6.0, 127, 7), (4, 6.03125, 128, 5), (4, 1.5, 125, 7), (8, 0.0, 27, 0), (4, 0.0, 27, 0),
                                              (8, 3.3e38, 246, 0x7E), (4, 3.3e38, 252, 7)])
def test_scales(bits, x, byte, code):
    row = np.zeros(128, np.float32)
    row[0] = x
    row = (row.view(np.uint32) >> 16).astype(np.uint16)
    codes, scales = encode(row, bits)
    assert scales.tolist() == [byte, 27, 27, 27] and codes[0] == code


def test_ties_go_to_the_even_code():
    row = np.zeros(128, np.float32)
    row[:4] = [6, 2.5, 3.5, 5]      # between 2 and 3, 3 and 4, 4 and 6
    row[32:36] = [448, 17, 19, 2.0 ** -10]   # between 16 and 18, 18 and 20, 0 and the least
    codes, scales = encode(bf16_bits(row), 4)
    assert decode(codes, scales, 4)[:4].tolist() == [6, 2, 4, 4]
    codes, scales = encode(bf16_bits(row), 8)
    assert decode(codes, scales, 8)[32:36].tolist() == [448, 16, 20, 0]


@pytest.mark.parametrize("bits", [8, 4])
def test_what_codes_stand_for_gets_the_same_codes(bits):
    rng = np.random.default_rng(bits)
    codes = rng.integers(0, 256, (50, 128 * bits // 8), dtype=np.uint8)
    codes[codes & 0x7F == 0x7F] = 0x7E if bits == 8 else 0x6E
    codes[:, ::32 * bits // 8] = 0x7E if bits == 8 else 0x77  # the largest in every group: the scale is then the same
    scales = rng.integers(100, 150, (50, 4)).astype(np.uint8)
    rows = bf16_bits(decode(codes, scales, bits))
    again, s = encode(rows, bits)
    assert np.array_equal(s, scales) and np.array_equal(again, codes)


def test_a_group_that_is_not_finite():
    row = np.zeros(128, np.uint16)
    row[40], row[100] = 0x7F80, 0xFFFF
    for bits in (8, 4):
        codes, scales = encode(row, bits)
        assert scales.tolist() == [27, 255, 27, 255]
        assert np.isnan(decode(codes, scales, bits)).tolist() == [False] * 32 + [True] * 32 + [False] * 32 + [True] * 32
