"""Which kernel a product of the gated feed-forward layer gets, and in how many slices (csrc/gated_plan.h, compiled for the CPU): the GPU
tests' sizes reach every kernel, a plan is well formed at any size, and choices whose times were measured are the fast ones.  And, in the
code that the compiler makes of csrc/gated_gemm.hip, nothing touches a transposing LDS read in flight."""
import ctypes
import os
import random
import re
import shutil
import subprocess

import pytest

from test_attention_reads_cpu import assembly, functions, unsafe

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_04802_amd", "csrc")
ASK = r"""
#include "gated_plan.h"
using namespace reslim;
extern "C" int choose(int M, int N, int cols, int slabs, int epi, int sliceable, int e4m3, double other, int *slices) {
  const GatedChoice c = gated_choose(M, N, cols, slabs, static_cast<GemmEpi>(epi), 256, sliceable, e4m3, other);
  *slices = c.slices;
  return c.us > 0 ? c.kernel : -1;
}
extern "C" int whole(int M, int N, int slabs) { return gated_whole_rounds(M, N, slabs, kEpiAct, 256); }
"""
RING, SMALL, WIDE, TALL = 1, 2, 3, 4      # 64 x 64; one 128 x 128 tile a work-group; persistent 256 x 256; 128 x 256
ACT, GELU, TWO, F32, STREAM = range(5)


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    cc = shutil.which("g++") or pytest.skip("no g++")
    d = tmp_path_factory.mktemp("plan")
    (d / "ask.cpp").write_text(ASK)
    subprocess.run([cc, "-O2", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(d / "ask.cpp"), "-o", str(d / "ask.so")], check=True)
    lib = ctypes.CDLL(str(d / "ask.so"))
    lib.choose.argtypes = [ctypes.c_int] * 7 + [ctypes.c_double, ctypes.POINTER(ctypes.c_int)]

    def ask(M, N, cols, slabs, epi, sliceable=False, e4m3=False, other=0.0):
        s = ctypes.c_int(0)
        return lib.choose(M, N, cols, slabs, epi, sliceable, e4m3, other, ctypes.byref(s)), s.value

    ask.whole = lib.whole
    return ask


def _products(ask, M, D, R):
    copy = 4e-6 / 4.5 * D * R
    e4m3 = {"in, e4m3": ask(M, 2 * R, R, D // 128, GELU, e4m3=True)} if D % 128 == 0 else {}
    return {**e4m3, "in": ask(M, 2 * R, R, D // 64, GELU), "in, kept": ask(M, 2 * R, R, D // 64, TWO),
            "out": ask(M, D, D, R // 64, ACT, True), "dgate": ask(M, R, 2 * R, D // 64, STREAM, other=2.0 + copy), "dx": ask(M, D, D, 2 * R // 64, ACT, True, other=2.0 + 2 * copy)}


def _sizes(name):
    text = open(os.path.join(ROOT, "tests", "test_gpu_gated_mlp.py")).read()
    return eval(re.search(name + r" = (\[.*?\])\n", text, re.S).group(1))


def test_the_gpu_tests_reach_every_kernel(choose):
    met = {}
    for M, D, R in _sizes("SIZES") + _sizes("LARGE"):
        for n, c in _products(choose, M, D, R).items():
            met.setdefault(n, set()).add((c[0], c[1] > 1))
    for n in ("in", "in, kept"):
        assert {k for k, _ in met[n]} == {RING, SMALL, WIDE, TALL}, (n, met[n])
    assert {k for k, _ in met["in, e4m3"]} == {RING, WIDE, TALL}
    assert {(RING, False), (RING, True), (SMALL, True)} <= met["out"], met["out"]
    assert {k for k, _ in met["dgate"]} == {RING, SMALL, WIDE, TALL}, met["dgate"]
    assert {(RING, False), (RING, True), (SMALL, True)} <= met["dx"] and {k for k, _ in met["dx"]} & {WIDE, TALL}, met["dx"]


@pytest.mark.parametrize("M", [2 ** 30 // 3, 2 ** 30, 2_000_000_000])
def test_a_product_that_no_launch_holds_in_tiles_is_persistent(choose, M):
    for D in (64, 128, 1024):
        for n, (kernel, slices) in _products(choose, M, D, 64).items():
            side, columns = 64 if kernel == RING else 128, 2 * 64 if n.startswith("in") else D if n in ("out", "dx") else 64
            assert kernel in (WIDE, TALL) or -(-M // side) * -(-columns // side) * slices <= 2 ** 23, (n, kernel)


def test_a_plan_is_well_formed_at_any_size(choose):
    r = random.Random(1)
    for _ in range(3000):
        M, N, slabs = int(2 ** r.uniform(0, 23)), 64 * int(2 ** r.uniform(0, 11)), int(2 ** r.uniform(0, 11))
        for sliceable in (False, True):
            for e4m3 in (False, True):
                k, s = choose(M, N, N, slabs, r.choice([ACT, GELU, TWO, STREAM]), sliceable, e4m3, r.choice([0.0, 50.0]))
                assert k in (RING, SMALL, WIDE, TALL) and 1 <= s <= 32 and (k != SMALL or not e4m3 or s > 1)
                if s > 1:      # every slice has a slab, and no fewer than four on average
                    per = -(-slabs // s)
                    assert sliceable and k in (RING, SMALL) and -(-slabs // per) == s and per >= 4


def test_measured_choices(choose):
    """Forward of both products with cold weights, microseconds (MI355X): 64 rows at 4096 x 10,944 72 with the ring and slices, 91 with 128 x 128 slices behind
    a persistent kernel, 196 without slices; 1000 rows 279 with two slices, 312 without; 2000 rows 423 without, 487 with two."""
    assert _products(choose, 64, 4096, 10944)["in"][0] == RING and _products(choose, 64, 4096, 10944)["out"][1] > 1
    assert _products(choose, 1000, 4096, 10944)["out"] == (SMALL, 2)
    assert _products(choose, 2000, 4096, 10944)["out"][1] == 1 and _products(choose, 20000, 4096, 10944)["in"] == (WIDE, 1)
    # gradients of 16 rows: 144 us where the weights are read as they lie, 455 with transposed copies; of 4000 rows 1870 with, 2440 without
    assert _products(choose, 16, 4096, 10944)["dx"][0] == _products(choose, 16, 4096, 10944)["dgate"][0] == RING
    assert _products(choose, 4000, 4096, 10944)["dx"][0] != RING


def test_nothing_touches_a_read_in_flight():
    kernels = 0
    for name, lines in functions(assembly("gated_gemm.hip")):
        groups, touched, open_ends = unsafe(lines)
        kernels += groups > 0
        assert not touched and not open_ends, (name, touched[:3], open_ends)
        # a ring kernel waits for its slab by count, never for all loads in flight inside the loop's steady state: one full wait before the epilogue
        if "gemm_ring_kernel" in name:
            assert any("vmcnt(8)" in l for l in lines), name
    assert kernels == 4          # dx whole and in slices, and the gate gradient with either activation


def test_rows_of_whole_rounds(choose):
    """The split is at a whole number of 256 x 256 tiles' rounds, and is made where it was measured to pay."""
    r = random.Random(2)
    split = 0
    for _ in range(4000):
        M, N, slabs = int(2 ** r.uniform(8, 18)), 64 * int(2 ** r.uniform(0, 8)), int(2 ** r.uniform(0, 8))
        rows = choose.whole(M, N, slabs)
        assert 0 < rows <= M
        if rows < M:
            split += 1
            assert rows % 256 == 0 and rows // 256 * -(-N // 256) <= -(-M // 256) * -(-N // 256) // 256 * 256
    assert split > 20
    for rows, K, kernel in ((16500, 1024, RING), (18000, 1024, SMALL), (16500, 2048, RING), (18000, 2048, SMALL), (20000, 2048, TALL)):      # the GPU test's
        assert choose.whole(rows, 2048, K // 64) == 16384 and choose(rows - 16384, 2048, 2048, K // 64, ACT)[0] == kernel
    # products of the layer's output map, microseconds of the layer in one launch and in two: 40,352 x 1024 x 2752 588 and 576, 17,000 x 2048 x 8192 1373 and
    # 1276, 20,000 x 2048 x 5504 1053 and 1034; the last two: within the noise
    for (M, N, K), pays in {(40352, 1024, 2752): True, (17000, 2048, 8192): True, (20000, 2048, 5504): True, (80704, 1024, 2752): False, (80704, 1536, 2752): False}.items():
        assert (choose.whole(M, N, K // 64) < M) == pays, (M, N, K)
