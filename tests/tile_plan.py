"""Which workgroups the library's rule takes for a call: csrc/tile_plan.h, built by the host's compiler, so that tests can say which programs their sizes run."""

import collections
import ctypes as C
import functools
import os
import shutil
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include "tile_plan.h"
using namespace slkv;
extern "C" int tile_shape(int i, int* wq, int* wk) { *wq = kTileShapes[i].wq; *wk = kTileShapes[i].wk; return kTileShapeCount; }
extern "C" int tile_has_shape(int dtype, int d, int i) { return has_shape(dtype, d, i); }
extern "C" void tile_prompt(const slkv_prompt_desc* d, int64_t* out) {
  const PromptPlan p = plan_prompt(d);
  out[0] = p.shape, out[1] = p.split, out[2] = p.slots, out[3] = 1, out[4] = p.bytes;
  for (int64_t b = 0; b < d->B; b += kPromptSeqs) out[3] &= prompt_in_order(d, p, b);
}
extern "C" void tile_tree(const slkv_cache_desc* d, int T, int64_t* out) {
  const TreePlan p = plan_tree(d, T);
  out[0] = p.shape, out[1] = p.split, out[2] = p.slots, out[3] = 1, out[4] = p.bytes;
}
"""

# waves of a workgroup along the queries and along the keys; whether keys are split into parts; workgroups of the largest launch; whether tiles come sequence by sequence in all launches
Plan = collections.namedtuple("Plan", "waves split blocks in_order workspace")


@functools.lru_cache(None)
def lib():
    compiler = shutil.which("g++") or shutil.which("clang++") or "/opt/rocm/llvm/bin/clang++"
    folder = tempfile.mkdtemp()
    try:
        with open(os.path.join(folder, "plan.cpp"), "w") as f:
            f.write(SOURCE)
        path = os.path.join(folder, "plan.so")
        subprocess.run([compiler, "-O1", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2508_15806_amd", "csrc"),
                        os.path.join(folder, "plan.cpp"), "-o", path], check=True)
        return C.CDLL(path)
    finally:
        shutil.rmtree(folder)


def shapes():
    """[(waves along the queries, along the keys)] of all shapes."""
    wq, wk = C.c_int(0), C.c_int(0)
    n = lib().tile_shape(0, C.byref(wq), C.byref(wk))
    found = []
    for i in range(n):
        lib().tile_shape(i, C.byref(wq), C.byref(wk))
        found.append((wq.value, wk.value))
    return found


def has_shape(dtype, d, i):
    return bool(lib().tile_has_shape(dtype, d, i))


def _plan(out):
    return Plan(shapes()[out[0]], bool(out[1]), out[2], bool(out[3]), out[4])


def prompt(batch):
    """Of a binding.PromptBatch."""
    out = (C.c_int64 * 5)()
    lib().tile_prompt(C.c_void_p(batch.address), out)
    return _plan(out)


def tree(layout, T):
    """Of a binding.CacheLayout and T drafted tokens."""
    out = (C.c_int64 * 5)()
    lib().tile_tree(C.c_void_p(layout.address), T, out)
    return _plan(out)
