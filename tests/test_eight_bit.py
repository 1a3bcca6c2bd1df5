"""The plain definitions of tests/eight_bit.py, at values worked out by hand, and refusals that need no GPU."""
import ctypes

import numpy as np
import pytest
import torch

import tests.eight_bit as eb
from paper_2410_09687_amd import moin


def test_codes_by_hand():
    #            0     1     1.125  1.0625 (tie: even)  1.1875 (tie)  448   464 (clamped)  2^-9  2^-10 (tie: 0)  3 * 2^-10 (tie: 2 * 2^-9)
    x = np.array([0.0, 1.0, 1.125, 1.0625, 1.1875, 448, 464, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10])
    want = [0, 1, 1.125, 1, 1.25, 448, 448, 2.0 ** -9, 0, 2.0 ** -8]
    assert eb.VALUES[eb.e4m3(x)].tolist() == want and eb.VALUES[eb.e4m3(-x)].tolist() == [-w for w in want]
    assert eb.e4m3(1.0) == 0x38 and eb.e4m3(448.0) == 0x7E and np.isnan(eb.VALUES[0x7F])
    fine = eb.VALUES[~np.isnan(eb.VALUES)]
    assert np.array_equal(eb.VALUES[eb.e4m3(fine)], fine)


@pytest.mark.parametrize("top,unit", [(448, 1), (463.9, 1), (464, 2), (928, 4), (1, 2.0 ** -8), (1.8125, 2.0 ** -7), (1.81, 2.0 ** -8), (0, 2.0 ** -117),
                                      (2.0 ** -130, 2.0 ** -117), (3.3e38, 2.0 ** 119)])
def test_scales_by_hand(top, unit):
    assert eb.power(eb.scale_byte(top)) == unit


def test_a_block_grows_and_its_codes_with_it():
    c = eb.Cache(np.full((1, 64 * 128 + 128), 0xFF), 1, 1, 64, 64)
    k = np.zeros((3, 1, 64))
    k[0, 0, 0], k[0, 0, 1], k[1, 0, 0], k[2, 0, 0] = 1.0, 2.0 ** -16, 448.0, 2.0
    c.append(k[:1], k[:1], [0, 1], [0])
    assert c.data[0, 64 * 128] == 119 and c.values()[0][0, 0, :2].tolist() == [1.0, 2.0 ** -16]
    c.append(k[1:], k[1:], [0, 2], [1, 2])
    v = c.values()
    assert c.data[0, 64 * 128] == 127 and v[0][:3, 0, 0].tolist() == [1, 448, 2] and v[1][0, 0, :2].tolist() == [1, 0]
    assert np.isnan(v[0][3]).all()       # beyond the tokens: as it was


def test_rotation_by_hand():
    x = np.array([[[1.0, 2.0, 3.0, 4.0]]])
    f = np.array([np.pi / 2, np.pi])
    assert np.allclose(eb.norm_rope(x, [1], f, None, 1, False, False)[0], [[[-3, -2, 1, -4]]])
    assert np.allclose(eb.norm_rope(x, [1], f, None, 1, False, True)[0], [[[-2, 1, -3, -4]]])
    assert np.allclose(eb.norm_rope(x, None, None, np.full(4, 2.0), 0.5, True, False)[0], 2 * x / np.sqrt(8.0))


def test_integers_by_hand():
    q, s = eb.integers(np.array([[127.0, 0.5, 1.5, -2.5], [0, 0, 0, 0], [1, np.inf, 0, 0]]))
    assert q[0].tolist() == [127, 0, 2, -2] and s[0] == 1 and q[1].tolist() == [0] * 4 and s[1] == 2.0 ** -126 and np.isnan(s[2])


def test_sizes():
    assert moin.KV8Pages.page_bytes(1, 64) == 64 * 128 + 128 and moin.KV8Pages.page_bytes(8, 128, 256) == 8 * 4 * 128 * 128 + 128
    assert moin.KV8Pages.page_bytes(100, 64, 128) == 100 * 2 * 128 * 64 + 512
    lib = moin.load()
    assert [lib.moin_i8_pitch(n) for n in (8, 256, 264, 1000, 2048, 131072)] == [256, 256, 384, 1024, 2048, 131072]
    assert [lib.moin_i8_pitch(n) for n in (0, -8, 12, 131080)] == [0] * 4
    for bad in ((32, 1, 64), (64, 0, 64), (64, 1, 96), (512, 1, 64)):
        assert lib.moin_kv8_page_bytes(*bad) == 0


def test_python_refusals():
    with pytest.raises(ValueError):
        moin.KV8Pages(torch.zeros(100, dtype=torch.uint8), 1, 64)
    with pytest.raises(ValueError):
        moin.KV8Pages.empty(1, 1, 96, device="cpu")
    with pytest.raises(ValueError):
        moin.I8Weight(torch.zeros((4, 200), dtype=torch.int8), torch.zeros(4), 200)
    with pytest.raises(ValueError):
        moin.I8Weight(torch.zeros((4, 256), dtype=torch.int8), torch.zeros(3), 200)
    with pytest.raises(ValueError):
        moin.I8Weight(torch.zeros((4, 256), dtype=torch.uint8), torch.zeros(4), 200)


def test_null_contexts_are_refused():
    lib = moin.load()
    p = moin._KVPagesStruct(None, 1, 64, 1, 64)
    assert lib.moin_kv8_append(None, ctypes.byref(p), None, None, 64, 64, 1, None, 1, None, None) == -1
    assert lib.moin_kv8_gather(None, ctypes.byref(p), None, 1, None, None, None) == -1
    assert lib.moin_kv8_attention(None, None, ctypes.byref(p), None, 64, 1, None, 1, 1.0, 0, None, 1, None, None) == -1
    assert lib.moin_qk_norm_rope(None, None, None, 1, 64, 64, 1, 1, 1, 64, None, None, 0, 0, None, None, 1.0, None, None, 64, 64, None) == -1
    assert lib.moin_i8_quantize(None, None, 1, 8, None, None, None) == -1
    assert lib.moin_i8_linear(None, None, 1, None, None, 8, 8, None, 1, None) == -1
    assert lib.moin_lora_linear_i8_planned(None, None, None, None, None, None, None, 8, 8, 0, 1.0, None, 1, None) == -1
