"""The plain definitions of tests/four_bit.py, at values worked out by hand (no GPU)."""
import numpy as np

import tests.four_bit as fb


def test_levels_and_scales_by_hand():
    x = np.zeros((1, 32))
    x[0, :6] = [6, -3.5, 0.25, 0.75, 5, 2.5]             # the largest is 6: unit 1; ties go to the even code: 4, 0, 1, 4, 2
    codes, E = fb.quantise(x)
    assert E[0] == 127
    assert fb.dequantise(codes, E)[0, :6].tolist() == [6, -4, 0, 1, 4, 2]
    for top, unit in [(6.9, 1), (7, 2), (8, 2), (14, 4), (3.4, 0.5), (3.5, 1), (2.0 ** -130, 2.0 ** -125), (3.3e38, 2.0 ** 125)]:
        x = np.zeros((1, 32))
        x[0, 3] = top
        assert 2.0 ** (int(fb.quantise(x)[1][0]) - 127) == unit, top
    assert fb.quantise(np.zeros((1, 32)))[1][0] == 127
    x[0, 5] = np.inf
    assert fb.quantise(x)[1][0] == 255 and np.isnan(fb.held(x)).all()


def test_plan_by_hand():
    # pages of 4: request 0 has 3 tokens (page 9) and gets 2 (one new page), 1 gets 4 (one), 2 nothing
    table = [[9, -1, -1], [-1, -1, -1], [-1, -1, -1]]
    t, lens, off, slots, n_free, fault = fb.plan([3, 0, 0], [2, 4, 0], 6, 4, 4, table, [5, 7, 2], 3)
    assert t == [[9, 2, -1], [7, -1, -1], [-1, -1, -1]] and lens == [5, 4, 0] and off == [0, 2, 6, 6]
    assert slots == [9 * 4 + 3, 2 * 4, 28, 29, 30, 31] and n_free == 1 and not fault
    # one free page: the second request is not served
    t, lens, _, slots, n_free, fault = fb.plan([3, 0, 0], [2, 4, 0], 6, 4, 4, table, [5], 1)
    assert t[0] == [9, 5, -1] and lens == [5, 0, 0] and slots[2:] == [-1] * 4 and n_free == 0 and fault


def test_attention_of_one_key_is_its_value():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(2, 4, 64)), rng.normal(size=(1, 2, 64)), rng.normal(size=(1, 2, 64))
    y, lse, _, _ = fb.attention(q, k, v, -1, 0.125, 0)   # the first token comes before the only key
    assert (y[0] == 0).all() and np.isneginf(lse[0]).all()
    assert np.allclose(y[1], np.repeat(v[0], 2, 0)) and np.allclose(lse[1], 0.125 * (q[1] * np.repeat(k[0], 2, 0)).sum(-1))
