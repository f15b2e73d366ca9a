"""The 8-bit attention's choices for a work list (csrc/kv8_plan.h, host arithmetic), for tests: compiled for the CPU on first use."""
import collections
import ctypes as C
import os
import subprocess
import tempfile

import paper_2402_18789_amd.binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """#include "kv8_plan.h"
extern "C" void plan(const flexco_maps* m, int nkv, int* out) {
  const flexco::Kv8Plan p = flexco::plan_kv8_attention(*m, nkv);
  out[0] = p.fold; out[1] = p.wavefronts; out[2] = p.whole;
}
"""
Plan = collections.namedtuple("Plan", "fold wavefronts whole")
MAX_PAGES = 512
_lib = None


def kv8_plan(maps, n_kv_heads):
    global _lib
    if _lib is None:
        with tempfile.TemporaryDirectory() as tmp:
            so = os.path.join(tmp, "plan.so")
            subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-shared", "-fPIC", "-x", "c++", "-I" + os.path.join(ROOT, "include"),
                            "-I" + os.path.join(ROOT, "paper_2402_18789_amd", "csrc"), "-", "-o", so], input=SOURCE, text=True, check=True)
            _lib = C.CDLL(so)
        _lib.plan.argtypes, _lib.plan.restype = [C.POINTER(B.Maps), C.c_int, C.POINTER(C.c_int)], None
    out = (C.c_int * 3)()
    _lib.plan(C.byref(maps), n_kv_heads, out)
    return Plan(out[0], out[1], bool(out[2]))


def pieces(maps, plan):
    """the most pieces that a request of one token is cut into"""
    return -(-maps.max_pages // (plan.fold * maps.kv_split_pages))
