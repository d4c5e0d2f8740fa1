"""The roundings that include/tfm_cache.h states for cached attention, from the formats themselves:
weights as half (11 bits) with 2^8 in front or as two halves, values as half with 2^7 in front."""

import os
import re

import numpy as np

from oracle import cache as oc

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include",
                      "tfm_cache.h")


def _weights():
    """float32 weights of at most 1, those next to the middle between two halves among them."""
    x = np.random.default_rng(0).uniform(0.5, 1, 1 << 14)
    near = (1024 + np.arange(1024) + 0.5)[:, None] + np.array([-1, 1]) * 2.0 ** -12
    x = np.concatenate([x, near.ravel() / 2048]).astype(np.float32)
    return np.concatenate([x * np.float32(2.0 ** -k) for k in range(40)])


def test_weights_as_halves():
    p = _weights()
    one = (p * 256).astype(np.float16)
    rest = (p * 256 - one.astype(np.float32)).astype(np.float16)
    off = np.abs(one.astype(np.float64) / 256 - p)
    two = np.abs((one.astype(np.float64) + rest.astype(np.float64)) / 256 - p)
    assert np.all(off <= np.maximum(2.0 ** -11 * p, 2.0 ** -33))
    assert np.any(off > np.maximum(2.0 ** -12 * p, 2.0 ** -33))          # no smaller power holds
    assert np.any(off > np.maximum(2.0 ** -11 * p, 2.0 ** -34))
    assert np.all(two <= np.maximum(2.0 ** -23 * p, 2.0 ** -33))
    text = re.sub(r"\s*\n \*\s*", " ", open(HEADER).read())
    said = re.search(r"to half \(by 2\^-(\d+) of each, or 2\^-(\d+) .*?two halves \(2\^-(\d+)\)", text)
    assert [int(x) for x in said.groups()] == [11, 33, 23]


def test_values_as_halves():
    for gap in range(97):
        x = oc.GRID * 2.0 ** (7 - gap)
        off = np.abs(x.astype(np.float16).astype(np.float64) - x).max()
        assert off == 0 if gap <= 22 else off <= 2.0 ** -40 * 448 * 2.0 ** 7, gap
