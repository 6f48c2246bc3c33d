"""Activations of the gated feed-forward layer's bf16 path (csrc/gate_act.h), compiled for the CPU, against 64 bits: the bounds that their comments
state, and what they give at the infinities."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
from scipy.special import erfc

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_04802_amd", "csrc")
# what the header takes from the device compiler; the median with a NaN is the smaller of the others
DEVICE = """#include <cmath>
#include <cstdint>
#define __device__
#define __forceinline__ inline
#define __builtin_amdgcn_exp2f exp2f
#define __builtin_amdgcn_rcpf(x) (1.0f / (x))
#define __builtin_amdgcn_fmed3f(a, lo, hi) fminf(fmaxf(a, lo), hi)
"""
MAIN = """#include "gate_act.h"
template <bool G> void all(const float *x, float *a, float *b, float *s, int n) {
  for (int i = 0; i < n; ++i) { a[i] = reslim::gate_act<G>(x[i]); reslim::gate_act_slope<G>(x[i], b[i], s[i]); }
}
extern "C" void ask(int gelu, const float *x, float *a, float *b, float *s, int n) { gelu ? all<true>(x, a, b, s, n) : all<false>(x, a, b, s, n); }
"""


@pytest.fixture(scope="module")
def act(tmp_path_factory):
    d = tmp_path_factory.mktemp("act")
    shutil.copy(os.path.join(CSRC, "gate_act.h"), d)
    (d / "common.h").write_text(DEVICE)
    (d / "main.cpp").write_text(MAIN)
    cxx = shutil.which("clang++") or "/opt/rocm/llvm/bin/clang++"
    subprocess.run([cxx, "-std=c++17", "-O1", "-ffp-contract=off", "-shared", "-fPIC", str(d / "main.cpp"), "-o", str(d / "act.so")], check=True)
    lib = ctypes.CDLL(str(d / "act.so"))

    def call(gelu, x):
        x = np.ascontiguousarray(x, np.float32)
        outs = [np.empty(len(x), np.float32) for _ in range(3)]
        lib.ask(int(gelu), *(t.ctypes.data_as(ctypes.c_void_p) for t in (x, *outs)), len(x))
        return [t.astype(np.float64) for t in outs]

    return call


X = np.concatenate([np.linspace(-30, 30, 600001), np.geomspace(1e-30, 1, 4001), -np.geomspace(1e-30, 1, 4001), [0.0, -0.0, 3e4, -3e4, 1e30, -1e30]]).astype(np.float32)


def test_gelu(act):
    x = X.astype(np.float64)
    cdf, pdf = 0.5 * erfc(-x / np.sqrt(2.0)), np.exp(-0.5 * x * x) / np.sqrt(2 * np.pi)
    a, b, s = act(True, X)
    assert np.array_equal(a, b)
    want, slope = x * cdf, cdf + x * pdf
    off = np.abs(a - want)
    inside = x >= -5
    assert (off[inside] <= 1.6e-5 * np.abs(want[inside])).all()                 # the fit, and rounding of fp32
    assert (off <= 1.7e-3 * np.abs(want) + 1e-36).all()                         # half a step of bf16 is 3.9e-3
    # the slope: the same error of the distribution, and v phi(v) with its exponent v^2 / (2 ln 2), rounded twice: v^2 2^-24 of it, and four roundings more
    tail = np.where(inside, 1.6e-5, 1.7e-3)
    assert (np.abs(s - slope) <= tail * cdf + 2.0 ** -24 * (x * x + 4) * np.abs(x) * pdf + 1e-36).all()
    # Phi(-15) = 3.7e-51, and fp32's smallest subnormal value is 1.4e-45 (Phi(-14) = 7.8e-45 is five of them)
    assert (s[(x < -5) & (x > -12)] < 0).all() and not np.any(a[x < -15]) and not np.any(s[x < -15])


def test_silu(act):
    x = X.astype(np.float64)
    with np.errstate(over="ignore"):
        p = 1.0 / (1.0 + np.exp(-x))
    a, b, s = act(False, X)
    assert np.array_equal(a, b)
    size = 2.0 ** -24 * (8 + 2 * np.abs(x))                                     # the exponent -x / ln 2 rounded, and a few more half steps
    assert (np.abs(a - x * p) <= size * np.abs(x * p) + 1e-35).all()            # below -88 the exponential leaves fp32 before 1 / it does
    assert (np.abs(s - (p + x * p * (1 - p))) <= size * (p + np.abs(x * p)) + 1e-35).all()


@pytest.mark.parametrize("gelu", [False, True])
def test_infinities_and_nan(act, gelu):
    a, b, s = act(gelu, [np.inf, -np.inf, np.nan])
    for t in (a, b):
        assert t[0] == np.inf and np.isnan(t[1:]).all()
    assert np.isnan(s).all()
