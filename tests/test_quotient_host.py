"""The quick quotients of the cache's quantiser (csrc/quotient.hpp), compiled for the host, over
everything that they may meet.  Powers of two apart the significands are all that matters:
far from the ends of the range every step scales exactly."""

import ctypes as C
import os
import subprocess

import numpy as np
import pytest

import paper_2608_15531_amd as fq

CSRC = os.path.join(os.path.dirname(fq.LIB_PATH), "csrc")

SHIM = r"""
#include "quotient.hpp"
extern "C" {
// how many a of n floats have quotient(a, b, 1 / b) != a / b
long wrong(const float* a, long n, float b) {
  long bad = 0;
  const float r = 1.f / b;
  for (long i = 0; i < n; ++i) bad += fqi::quotient(a[i], b, r) != a[i] / b;
  return bad;
}
float inverse(float s, float r0) { return fqi::inverse(s, r0); }
}
"""


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    d = tmp_path_factory.mktemp("quotient")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-O2", "-ffp-contract=off", "-std=c++17", "-fPIC", "-shared", "-I", CSRC, str(d / "shim.cpp"),
                    "-o", str(d / "shim.so")], check=True)
    s = C.CDLL(str(d / "shim.so"))
    s.wrong.argtypes = [C.c_void_p, C.c_long, C.c_float]
    s.wrong.restype = C.c_long
    s.inverse.argtypes = [C.c_float, C.c_float]
    s.inverse.restype = C.c_float
    return s


@pytest.mark.parametrize("top", [255.0, 15.0])
def test_spans_over_the_codes(shim, top):
    a = (np.arange(1 << 23, dtype=np.uint32) | np.uint32(0x3F800000)).view(np.float32)   # [1, 2)
    assert shim.wrong(a.ctypes.data, len(a), top) == 0
    for e in (-90, 90):   # the ends of the quick path
        b = a[::97] * np.float32(2.0 ** e)
        assert shim.wrong(b.ctypes.data, len(b), top) == 0


def test_values_over_scales(shim):
    a = (np.arange(128, 256) / 128).astype(np.float32)   # all significands of bf16
    both = np.concatenate([a, -a, a / 256, -a / 4, [np.float32(0)]]).astype(np.float32)
    for s in a:
        assert shim.wrong(both.ctypes.data, len(both), float(s)) == 0


def test_inverses_of_scales(shim):
    for s in (np.arange(128, 256) / 128).astype(np.float32):
        want = np.float32(1) / s
        for k in range(-2, 3):
            near = np.uint32(int(want.view(np.uint32)) + k).view(np.float32)
            assert np.float32(shim.inverse(float(s), float(near))) == want, (s, k)
