"""Pins of the float64 oracle of contexts kept in 8 bits (oracle/cache.py) and of adjusted logits."""

import numpy as np
import pytest

from oracle import cache as oc
from oracle import vocab


def test_codes_are_the_e4m3_values():
    torch = pytest.importorskip("torch")
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    got = oc.decode(codes)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    assert np.array_equal(got[ok], want[ok])
    back = oc.encode(got)
    assert np.array_equal(back[ok], codes[ok]) and np.all(back[~ok] == oc.NAN)


def test_encoding_is_the_nearest_value_ties_to_even():
    assert oc.encode([17.0, 19.0, -17.0, 448.0, 440.0, 2.0 ** -10, 3 * 2.0 ** -10]).tolist() == \
        oc.encode([16.0, 20.0, -16.0, 448.0, 448.0, 0.0, 2.0 ** -8]).tolist()
    rng = np.random.default_rng(0)
    x = rng.normal(size=2000) * 2.0 ** rng.integers(-10, 7, 2000)
    got = np.abs(oc.decode(oc.encode(x)) - x)
    best = np.abs(np.concatenate([oc.GRID, -oc.GRID])[None] - x[:, None]).min(1)
    assert np.array_equal(got, best)


def test_power_is_the_least_that_holds():
    assert oc.power([0.0]) == oc.E_MIN and oc.power([448.0]) == 127 and oc.power([449.0]) == 128
    assert oc.power([np.nan, np.inf, 1.0]) == oc.power([1.0])
    assert oc.power([1e30]) == oc.E_MIN and oc.power([448.0 * 2.0 ** 48]) == oc.E_MAX
    for x in (0.1, 3.0, 1e-20, 5e10):
        e = oc.power([x])
        assert x <= 448 * 2.0 ** (e - 127) and (e == oc.E_MIN or x > 448 * 2.0 ** (e - 128))


def _empty(n_pages, heads, page, d):
    return (np.full((n_pages, heads, page, d), 0x55, np.uint8),
            np.full((n_pages, heads, d, page), 0x66, np.uint8),
            np.full((n_pages, heads, 2), 0x77, np.uint8))


def test_appending_at_once_or_row_by_row_differs_only_by_the_second_rounding():
    """With rows of falling size the powers never grow and both ways give the same bytes."""
    rng = np.random.default_rng(1)
    k = rng.uniform(-1, 1, (1, 40, 2, 16))
    k[0, 0], k[0, 16], k[0, 32] = 1.0, 1.0, 1.0     # each block's largest first
    v = k[:, :, ::-1]
    a = oc.append(*_empty(3, 2, 16, 16), k, v, 3)
    b = _empty(3, 2, 16, 16)
    for i in range(40):
        b = oc.append(*b, k[:, i:i + 1], v[:, i:i + 1], 3, lens=[i])
    for x, y in zip(a, b):
        assert np.array_equal(x, y)
    assert np.all(a[0][2, :, 8:] == 0x55)            # rows behind the last, as they were


def test_growing_power_rounds_again():
    pool = oc.append(*_empty(1, 1, 16, 16), np.full((1, 1, 1, 16), 1.125), np.ones((1, 1, 1, 16)), 1)
    pool = oc.append(*pool, np.full((1, 1, 1, 16), 1e4), np.ones((1, 1, 1, 16)), 1, lens=[1])
    K, V, here = oc.rows_of(*pool, 1, None, 0, 2, 0)
    assert np.all(K[0] == 1.125) and np.all(np.abs(K[1] / 1e4 - 1) <= 2.0 ** -4) and here.all()
    pool = oc.append(*pool, np.full((1, 1, 1, 16), 1e12), np.ones((1, 1, 1, 16)), 1, lens=[2])
    assert np.all(oc.rows_of(*pool, 1, None, 0, 3, 0)[0][0] == 0)  # below the block's least code


def test_attention_by_hand():
    """One key: its value; equal keys: the mean; and against a plain softmax."""
    rng = np.random.default_rng(2)
    k, v = rng.normal(size=(2, 20, 1, 16)), rng.normal(size=(2, 20, 1, 16))
    pool = oc.append(*_empty(4, 1, 16, 16), k, v, 2)
    q = rng.normal(size=(2, 3, 2, 16))
    out, lse = oc.attend(q, *pool, 2, None, [1, 20], None, 0.3, True)[:2]
    assert np.all(lse[0, :2] == -np.inf) and not out[0, :2].any()
    V0 = oc.rows_of(*pool, 2, None, 0, 1, 0)[1]
    assert np.allclose(out[0, 2], V0[0])
    K, V, _ = oc.rows_of(*pool, 2, None, 1, 20, 0)
    for i in range(3):
        n = 20 - 3 + i + 1
        s = 0.3 * K[:n] @ q[1, i, 1]
        p = np.exp(s) / np.exp(s).sum()
        assert np.allclose(out[1, i, 1], p @ V[:n]) and np.isclose(lse[1, i, 1], np.log(np.exp(s).sum()))


def test_absent_pages_are_neither_written_nor_seen():
    rng = np.random.default_rng(3)
    k = rng.normal(size=(1, 48, 1, 16))
    pages = np.array([[2, -1, 0]])
    pool = oc.append(*_empty(3, 1, 16, 16), k, k, 3, pages)
    assert np.all(pool[0][1] == 0x55)
    q = rng.normal(size=(1, 1, 1, 16))
    a = oc.attend(q, *pool, 3, pages, [48], None, 1.0, False)
    b = oc.attend(q, *pool, 2, np.array([[2, 0]]), [32], None, 1.0, False)
    assert np.allclose(a[0], b[0]) and np.allclose(a[1], b[1])


def test_adjusted_logits_by_hand():
    s = [2.0, -2.0, 0.0, 5.0, np.nan, 1.0]
    x, _ = vocab.adjust_row(s, None, [0, 1, 1, 2, -1, 99], 2.0, 0.5, 0.25, [3, 3, 0, -7],
                            [10.0, 99.0, -1.0, 5.0], [0b111111])
    assert x[:4].tolist() == [1.0 - 0.75 - 1.0, -4.0 - 1.0, -0.75, 15.0]
    assert np.isnan(x[4]) and x[5] == 1.0
    x, _ = vocab.adjust_row(s, 5, allowed=[0b101001])
    assert x.tolist() == [2.0, -np.inf, -np.inf, 5.0, -np.inf, -np.inf]
    assert vocab.adjust_row([3.0], None, [0], 0.0)[0][0] == 3.0
