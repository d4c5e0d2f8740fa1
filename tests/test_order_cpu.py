"""The search for the smallest logit that min_p keeps (csrc/order.h), compiled for the host: right,
and never more than 64 tests of a key, however far the guess lies from the answer.  Where
top + log(min_p) temperature cancels, the keys between a guess and the answer are counted in
hundreds of millions: a walk from one to the next would keep a GPU busy for seconds."""

import ctypes
import math
import os
import subprocess

import numpy as np
import pytest

from paper_2606_03681_amd import build

SOURCE = """
#include "order.h"
extern "C" uint32_t key(float x) { return tfm::key_of(x); }
extern "C" float logit(uint32_t k) { return tfm::of_key(k); }
extern "C" uint32_t first(uint32_t lo, uint32_t hi, uint32_t guess, uint32_t answer, int* tests) {
  *tests = 0;
  return tfm::first_key(lo, hi, guess, [&](uint32_t k) {
    ++*tests;
    return k < lo || k > hi ? __builtin_trap(), false : k >= answer;
  });
}
extern "C" uint32_t min_p(double least, float tau, float top) {
  return tfm::min_p_key(least, tau, top);
}
"""


@pytest.fixture(scope="module")
def order(tmp_path_factory):
    where = tmp_path_factory.mktemp("order")
    src, lib = str(where / "order.hip"), str(where / "order.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run([build.HIPCC, "-O2", "-std=c++17", "-fPIC", "-shared", "--offload-host-only",
                    "-x", "hip", f"-I{build.CSRC}", src, "-o", lib], check=True,
                   capture_output=True, text=True)
    L = ctypes.CDLL(lib)
    u32, f32, f64 = ctypes.c_uint32, ctypes.c_float, ctypes.c_double
    L.key.restype, L.key.argtypes = u32, [f32]
    L.logit.restype, L.logit.argtypes = f32, [u32]
    L.first.restype, L.first.argtypes = u32, [u32, u32, u32, u32, ctypes.POINTER(ctypes.c_int)]
    L.min_p.restype, L.min_p.argtypes = u32, [f64, f32, f32]
    return L


def test_keys_keep_the_order_of_the_logits(order):
    big = float(np.finfo(np.float32).max)
    x = [-big, -1.5, -1e-45, 0.0, 1e-45, 2e-42, 1.0, big, math.inf]
    keys = [order.key(v) for v in x]
    assert keys == sorted(set(keys)) and keys[0] == 0x00800000
    assert [order.logit(k) for k in keys] == [float(np.float32(v)) for v in x]
    assert order.key(-0.0) == order.key(0.0)
    assert order.key(-math.inf) == order.key(math.nan) == 0


def test_search_takes_few_tests_from_any_guess(order):
    rng = np.random.default_rng(0)
    lo0, hi0 = 0x00800000, 0xff800000
    ends = [(lo0, hi0), (lo0, lo0), (hi0, hi0), (lo0, lo0 + 1), (5, 9)]
    ends += [tuple(sorted(rng.integers(lo0, hi0, 2).tolist())) for _ in range(200)]
    tests = ctypes.c_int()
    for lo, hi in ends:
        some = [lo, hi, lo + (hi - lo) // 2] + rng.integers(lo, hi + 1, 6).tolist()
        some += [min(max(a + d, lo), hi) for a in some[:4] for d in (-2, -1, 1, 2)]
        for guess in some:
            for answer in some:
                assert order.first(lo, hi, guess, answer, ctypes.byref(tests)) == answer
                assert tests.value <= 64
                if abs(guess - answer) <= 2:
                    assert tests.value <= 5


# (top, temperature, min_p): ordinary ones, and ones whose border cancels to about 0 from either side
CANCEL = [(float.fromhex("0x1.485ff2p+0"), float.fromhex("0x1.1d3904p-1"), 0.1),
          (2.384186e-07, 1.0, 0.99999976), (math.log(10.0), 1.0, 0.1), (2 * math.log(4.0), 2.0, 0.25)]
ROWS = CANCEL + [(0.0, 1.0, 0.5), (3.7, 0.8, 0.02), (-3.7, 0.8, 0.02), (88.0, 1e-3, 1e-30),
                 (-1e30, 1.0, 0.5), (3.4e38, 3e38, 1e-30), (-3.4e38, 3e38, 0.3), (1.0, 1e-45, 0.1),
                 (1.0, math.inf, 0.1), (5.0, 1.0, 1.0), (1e-42, 1e-40, 0.7), (-0.0, 1.0, 1e-45)]


@pytest.mark.parametrize("top,tau,min_p", ROWS)
def test_smallest_kept_logit(order, top, tau, min_p):
    top, tau = float(np.float32(top)), float(np.float32(tau))
    least = math.log(float(np.float32(min_p)))

    def reaches(k):
        return (float(order.logit(k)) - top) * (1.0 / tau) >= least

    k = order.min_p(least, tau, top)
    assert 0x00800000 <= k <= order.key(top)
    assert reaches(k) and (k == 0x00800000 or not reaches(k - 1))


def test_smallest_kept_logit_next_to_infinity(order):
    assert order.min_p(math.log(0.5), 1.0, math.inf) == order.key(math.inf)
