"""Which kernels an entry point of the library launches, without a GPU: a stand-in for the HIP runtime, found before the real one because it is
loaded first, notes every launch (kernel, grid) and runs none.  Work goes to a process of its own, where torch is not imported."""
import json
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STAND_IN = r"""
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cxxabi.h>
#include <map>
#include <string>
#include <vector>
struct Dim { uint32_t x, y, z; };
static std::map<const void *, std::string> names;
static std::vector<std::string> launches;
static std::string text;
static Dim grid, block;
static size_t shared;
static void *stream;
static int cus = 256, device_error = 0, attribute_error = 0;
extern "C" {
void **__hipRegisterFatBinary(const void *) { static void *h; return &h; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
void __hipRegisterFunction(void **, const void *f, char *, const char *name, unsigned, void *, void *, void *, void *, int *) {
  int bad = 0;
  char *s = abi::__cxa_demangle(name, nullptr, nullptr, &bad);
  names[f] = bad ? name : s;
  std::free(s);
}
int __hipPushCallConfiguration(Dim g, Dim b, size_t s, void *q) { grid = g; block = b; shared = s; stream = q; return 0; }
int __hipPopCallConfiguration(Dim *g, Dim *b, size_t *s, void **q) { *g = grid; *b = block; *s = shared; *q = stream; return 0; }
int hipLaunchKernel(const void *f, Dim g, Dim, void **, size_t, void *) {
  char at[64];
  std::snprintf(at, sizeof at, "|%u %u %u", g.x, g.y, g.z);
  launches.push_back(names[f] + at);
  return 0;
}
int hipGetLastError() { return 0; }
const char *hipGetErrorString(int) { return "error of the stand-in"; }
int hipGetDevice(int *d) { *d = 0; return device_error; }
int hipDeviceGetAttribute(int *v, int, int) { *v = cus; return 0; }
int hipFuncSetAttribute(const void *, int, int) { return attribute_error; }
int hipGetSymbolAddress(void **p, const void *) { *p = reinterpret_cast<void *>(1 << 20); return 0; }
void stand_in(int units, int device, int attribute) { cus = units; device_error = device; attribute_error = attribute; }
const char *stand_in_launches() {
  text.clear();
  for (const std::string &l : launches) text += l + "\n";
  launches.clear();
  return text.c_str();
}
}
"""
# what the asking code finds: lib, B (binding), p (an address that nothing follows), launches() -> [(kernel, (x, y, z))], out (a list to be handed back)
PROLOGUE = """
import ctypes as C, json, sys
s = C.CDLL({stand_in!r}, mode=C.RTLD_GLOBAL)
s.stand_in_launches.restype = C.c_char_p
sys.path.insert(0, {root!r})
from paper_2505_04802_amd import binding as B
lib, p, out = B.load(), 1 << 20, []
def launches():
    pairs = [l.rsplit("|", 1) for l in s.stand_in_launches().decode().splitlines()]
    return [(k.replace("reslim::", "").replace("gated::", "").replace("(anonymous namespace)::", ""), tuple(int(n) for n in g.split())) for k, g in pairs]
def gated_weights(**kw):
    return C.byref(B.GatedMlpWeightsC(**{{"w_in": p, "w_out": p, **kw}}))
GRADS = C.byref(B.GatedMlpGradsC(w_in=p, b_in=p, w_out=p, b_out=p))
"""
_built = {}


def ask(tmp_path_factory, code: str, **given):
    """Runs `code` beside the stand-in; `given` are plain values it finds under their names.  Returns what it appended to `out`."""
    if "at" not in _built:
        cc = shutil.which("g++") or pytest.skip("no g++")
        d = tmp_path_factory.mktemp("stand_in")
        (d / "stand_in.cpp").write_text(STAND_IN)
        subprocess.run([cc, "-O1", "-std=c++17", "-shared", "-fPIC", str(d / "stand_in.cpp"), "-o", str(d / "stand_in.so")], check=True)
        _built["at"] = str(d / "stand_in.so")
    text = PROLOGUE.format(stand_in=_built["at"], root=ROOT) + "".join(f"{n} = json.loads({json.dumps(v)!r})\n" for n, v in given.items()) + code + "\nprint(json.dumps(out), flush=True)\n"
    r = subprocess.run([sys.executable, "-c", text], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    return json.loads(r.stdout.splitlines()[-1])
