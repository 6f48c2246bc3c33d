"""What the gated feed-forward layer launches (a stand-in for the HIP runtime notes it; nothing runs) against what csrc/gated_plan.h plans."""
import ctypes
import os
import random
import re
import shutil
import subprocess

import pytest

from launch_record import ask

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_04802_amd", "csrc")
PLAN = r"""
#include "gated_plan.h"
using namespace reslim;
extern "C" int choose(int M, int N, int slabs, int sliceable, double other, int *slices) {
  const GatedChoice c = gated_choose(M, N, N, slabs, kEpiAct, 256, sliceable, false, other);
  *slices = c.slices;
  return c.kernel;
}
extern "C" int whole(int M, int N, int slabs) { return gated_whole_rounds(M, N, slabs, kEpiAct, 256); }
"""
RING, SMALL, WIDE, TALL = 1, 2, 3, 4
CALLS = """
for M, D, R in sizes:
    rc = [lib.reslim_gated_mlp_fwd(p, None, gated_weights(), 0, M, D, R, 1, p, p, 1 << 40, None)]
    fwd = launches()
    rc.append(lib.reslim_gated_mlp_bwd(p, p, p, p, gated_weights(), 0, M, D, R, 1, 1, p, GRADS, p, 1 << 40, None))
    out.append((rc, fwd, launches()))
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cc = shutil.which("g++") or pytest.skip("no g++")
    d = tmp_path_factory.mktemp("plan")
    (d / "ask.cpp").write_text(PLAN)
    subprocess.run([cc, "-O2", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(d / "ask.cpp"), "-o", str(d / "ask.so")], check=True)
    lib = ctypes.CDLL(str(d / "ask.so"))
    lib.choose.argtypes = [ctypes.c_int] * 4 + [ctypes.c_double, ctypes.POINTER(ctypes.c_int)]

    def planned(M, N, K, other):
        """[(kernel, slices, rows)] of one product."""
        s = ctypes.c_int(0)
        kernel = lib.choose(M, N, K // 64, 1, other, ctypes.byref(s))
        rows = lib.whole(M, N, K // 64) if kernel == WIDE else M
        if rows == M:
            return [(kernel, s.value, M)]
        return [(WIDE, 1, rows), (lib.choose(M - rows, N, K // 64, 0, 0.0, ctypes.byref(s)), 1, M - rows)]

    return planned


def _products(launched):
    """[(kernel, slices)] of the products with plain or sliced results among the launches: epilogues 0 and 96."""
    found = []
    for name, grid in launched:
        m = re.match(r"void (gemm_ring_kernel|gemm_bf16_pp_kernel|gemm_bf16_kernel)<(.*?)>", name)
        if not m:
            continue
        args = [int(a) if a.strip().isdigit() else a.strip() for a in m[2].split(",")]
        epi = args[0] if m[1] == "gemm_ring_kernel" else args[-1]
        if epi in (0, 96):
            found.append((RING if m[1] == "gemm_ring_kernel" else SMALL if m[1] == "gemm_bf16_kernel" else {2: WIDE, 1: TALL}[args[0]], grid[1]))
    return found


def _sizes():
    r, sizes = random.Random(3), [(16500, 2048, 1024), (18000, 2048, 1024), (20000, 2048, 1024), (2323, 1344, 3840), (1448, 2112, 4864), (1431, 2368, 1728), (40352, 1024, 2752)]
    while len(sizes) < 1500:
        M, D, R = int(2 ** r.uniform(0, 16.5)), 64 * int(2 ** r.uniform(0, 6)), 64 * int(2 ** r.uniform(0, 7.5))
        if M * D * R < 2e12:
            sizes.append((M, D, R))
    return sizes


def test_the_planned_kernels_are_launched(plan, tmp_path_factory):
    sizes, kinds = _sizes(), {"out": set(), "dx": set()}
    for (M, D, R), (rc, fwd, bwd) in zip(sizes, ask(tmp_path_factory, CALLS, sizes=sizes)):
        assert rc == [0, 0]
        copy = 4e-6 / 4.5 * D * R
        for what, launched, want in (("out", fwd, plan(M, D, R, 0.0)), ("dx", bwd, plan(M, D, 2 * R, 2.0 + 2 * copy))):
            assert _products(launched) == [(k, s) for k, s, _ in want], (what, M, D, R, want)
            kinds[what].add((want[0][0], want[0][1] > 1, len(want), want[-1][0]))
    for what, met in kinds.items():      # whole products of every kernel, slices, and rows of a last round
        assert {(RING, True, 1, RING), (SMALL, True, 1, SMALL), (SMALL, False, 1, SMALL), (WIDE, False, 1, WIDE), (TALL, False, 1, TALL)} <= met, (what, met)
        assert any(n == 2 for _, _, n, _ in met), (what, met)


UNITS = """
s.stand_in(512, 0, 0)                                   # the process meets a device of 512 compute units in this call
out.append(lib.reslim_gated_mlp_fwd(p, None, gated_weights(), 0, *size, 1, p, p, small, None) if train == 0 else
           lib.reslim_gated_mlp_fwd_train(p, gated_weights(), 0, *size, 1, p, p, p, p, small, None))
out.append(launches())
n = C.c_size_t(0)
out.append(lib.reslim_gated_mlp_workspace_bytes(*size, 1, C.byref(n)))
out.append(n.value)
out.append(lib.reslim_gated_mlp_fwd(p, None, gated_weights(), 0, *size, 1, p, p, n.value, None))
out.append(len(launches()))
out.append(lib.reslim_gated_mlp_fwd(p, None, gated_weights(), 0, *size, 1, p, p, n.value - 1, None))
out.append(len(launches()))
"""


@pytest.mark.parametrize("train", [0, 1])
def test_a_workspace_is_checked_for_the_device_that_the_call_meets(tmp_path_factory, train):
    """Twice the compute units, more slices of the output map: the size that was right for 256 is refused, before anything is enqueued."""
    M, D, R = size = (128, 1024, 8192)
    with_256 = ask(tmp_path_factory, "n = C.c_size_t(0)\nlib.reslim_gated_mlp_workspace_bytes(*size, 1, C.byref(n))\nout.append(n.value)", size=size)[0]
    refused, nothing, ok, need, ran, launches, short, none = ask(tmp_path_factory, UNITS, size=size, small=with_256, train=train)
    assert need > with_256
    assert refused == -5 and nothing == [] and ok == 0 and ran == 0 and launches == 3 and short == -5 and none == 0


@pytest.mark.parametrize("device,attribute,code", [(100, 0, 0), (1, 0, -4), (0, 1, -4)], ids=["no device", "device error", "attribute error"])
def test_workspace_queries_report_errors(tmp_path_factory, device, attribute, code):
    """Without a device the sizes are those of 256 compute units; any other error is the call's."""
    got = ask(tmp_path_factory, """
s.stand_in(64, device, attribute)
for query in (lambda n: lib.reslim_gated_mlp_workspace_bytes(128, 1024, 8192, 1, n), lambda n: lib.reslim_gated_mlp_bwd_workspace_bytes(128, 1024, 8192, 1, 1, n)):
    n = C.c_size_t(0)
    out.append([query(C.byref(n)), n.value, lib.reslim_last_error(None).decode() if want else ""])
out.append([lib.reslim_gated_mlp_workspace_bytes(128, 1024, 8192, 0, C.byref(n)), n.value, ""])      # fp32 asks no device
""", device=device, attribute=attribute, want=code)
    assert [g[0] for g in got] == [code, code, 0]
    assert all((g[1] > 0) == (g[0] == 0) for g in got)
    if code:
        assert all("workspace_bytes" in g[2] for g in got[:2])


def test_the_gpu_tests_of_few_fp32_rows_take_their_kernel(tmp_path_factory):
    text = open(os.path.join(os.path.dirname(os.path.abspath(__file__)), "test_gpu_gated_few_rows.py")).read()
    sizes, taken = (eval(re.search(r"^%s = (.*)$" % n, text, re.M).group(1)) for n in ("SIZES", "TAKEN"))
    got = ask(tmp_path_factory, """
for size in sizes:
    out.append([lib.reslim_gated_mlp_fwd(p, None, gated_weights(), gate, *size, 0, p, p, 1 << 40, None) for gate in (0, 1)])
    out.append([k for k, _ in launches() if "sum" not in k])
""", sizes=sizes)
    for size, want, rc, kernels in zip(sizes, taken, got[::2], got[1::2]):
        assert rc == [0, 0] and len(kernels) == 4
        for k, gelu in ((0, "false"), (2, "true")):
            assert tuple("gated_f32_few_kernel" in n for n in kernels[k:k + 2]) == want, (size, kernels)
            assert not want[0] or f"<2, {gelu}>" in kernels[k], kernels
            assert not want[1] or "<1, false>" in kernels[k + 1], kernels
    steps = {(k // 16 + 7) // 8 for s, t in zip(sizes, taken) for k, on in zip((s[1], s[2]), t) if on}
    assert {1, 2, 4, 5, 8, 17, 22} <= steps, steps      # steps a wave: fewer than, as many as and more than the four of a turn and the eight of two


def test_the_gpu_tests_of_cut_products_cut_them(tmp_path_factory):
    """In the whole calls the product is cut behind row 16,384, with each kernel for the rest; the parts are cut elsewhere or not at all, and none is sliced."""
    text = open(os.path.join(os.path.dirname(os.path.abspath(__file__)), "test_gpu_gated_cuts.py")).read()
    given = {"AT": 16384}
    for n in ("AT", "ROWS", "PARTS"):
        given[n] = eval(re.search(r"^%s = (.*?)(  #.*)?$" % n, text, re.M).group(1), {}, given)
    for what, R in (("out", 2048), ("dx", 1024)):
        calls = [(rows, None) for rows in given["ROWS"]] + [(rows, p) for rows in given["ROWS"] for p in given["PARTS"]]
        sizes = [(rows if p is None else len(range(rows)[slice(*p)]), 2048, R) for rows, p in calls]
        found = [_products(fwd if what == "out" else bwd) for _, fwd, bwd in ask(tmp_path_factory, CALLS, sizes=sizes)]
        assert found[:3] == [[(WIDE, 1), (k, 1)] for k in (RING, SMALL, TALL)], (what, found[:3])
        assert all(s == 1 for f in found for _, s in f), (what, found)
        whole = {k for f in found[3:] if len(f) == 1 for k, _ in f}
        assert {SMALL, WIDE, TALL} & whole == whole and len(whole) >= 2, (what, whole)


def test_the_gpu_tests_of_short_contractions_take_the_large_kernels(tmp_path_factory):
    text = open(os.path.join(os.path.dirname(os.path.abspath(__file__)), "test_gpu_gated_slabs.py")).read()
    e4m3, bf16 = (eval(re.search(r"^%s = (\[.*?\])" % n, text, re.M).group(1)) for n in ("E4M3", "BF16"))
    got = ask(tmp_path_factory, """
for size in e4m3:
    lib.reslim_gated_mlp_fwd(p, p, gated_weights(in_scale=p), 0, *size, 2, p, p, 1 << 40, None)
    out.append(launches()[0][0])
for size in bf16:
    lib.reslim_gated_mlp_bwd(p, p, p, p, gated_weights(), 0, *size, 1, 1, p, GRADS, p, 1 << 40, None)
    out.append([k for k, _ in launches() if ", 64>" in k or "<64, true>" in k][0])      # the hidden layer's gradient
""", e4m3=e4m3, bf16=bf16)
    assert ["gemm_bf16_pp_kernel<2, 36>" in got[0], "gemm_bf16_pp_kernel<2, 36>" in got[1], "gemm_bf16_pp_kernel<1, 36>" in got[2]] == [True] * 3, got
    assert all("gemm_bf16_kernel<128, 128" in k for k in got[4:6]) and "gemm_bf16_pp_kernel<2, 64>" in got[-1], got
