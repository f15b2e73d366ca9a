"""The host side of the 8-bit cache compiled on its own: its tests under AddressSanitizer and UndefinedBehaviorSanitizer, and no exception
past the C boundary where host memory runs out."""
import os
import subprocess
import sys

import pytest

from test_host_sanitized import ROOT, _build_module

OUT_OF_MEMORY = r"""
#include <cstdio>
#include <cstdlib>
#include <new>
#include "flexco_kv8_host.cpp"
static bool out_of_memory = false;
void* operator new(size_t n) {
  if (out_of_memory) throw std::bad_alloc();
  if (void* p = malloc(n)) return p;
  throw std::bad_alloc();
}
void operator delete(void* p) noexcept { free(p); }
void operator delete(void* p, size_t) noexcept { free(p); }
namespace flexco {
int32_t fail(int32_t code, const char*, ...) { return code; }
void clear_error() {}
}
int main() {
  int32_t slot[3] = {0, 17, 34}, pos[3] = {0, 1, 2}, req[3] = {0, 1, 2}, runs[6], n = -1;
  flexco_maps m = {};
  m.T = 3; m.n_req = 3; m.page_size = 16; m.slot = slot; m.tok_pos = pos; m.tok_req = req;
  const int32_t before = flexco_kv8_runs(&m, runs, 3, &n), found = n;
  n = -1;
  out_of_memory = true;
  const int32_t without = flexco_kv8_runs(&m, runs, 3, &n);
  out_of_memory = false;
  return before == FLEXCO_OK && found == 3 && without == FLEXCO_EWORKSPACE && n == -1 ? 0 : 1;
}
"""


def test_no_exception_passes_the_c_boundary(tmp_path):
    exe = str(tmp_path / "oom")
    include = ["-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_2402_18789_amd", "csrc")]
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-x", "c++"] + include + ["-", "-o", exe], input=OUT_OF_MEMORY, text=True, check=True)
    r = subprocess.run([exe], timeout=60, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]


def test_runs_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    lib = str(tmp_path / "libflexco_host_san.so")
    _build_module().build_host_sanitized(lib)
    asan = subprocess.run(["g++", "-print-file-name=libasan.so"], capture_output=True, text=True).stdout.strip()
    if not os.path.isabs(asan) or not os.path.exists(asan):
        pytest.skip("no shared AddressSanitizer runtime beside g++")
    env = dict(os.environ)
    env["LD_PRELOAD"] = asan + (":" + env["LD_PRELOAD"] if env.get("LD_PRELOAD") else "")
    env["FLEXCO_LIB_PATH"], env["FLEXCO_HOST_ONLY"] = lib, "1"
    env["ASAN_OPTIONS"] = "detect_leaks=0:abort_on_error=1"
    env["UBSAN_OPTIONS"] = "halt_on_error=1:print_stacktrace=1"
    cmd = [sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", "tests/test_kv8_host.py", "tests/test_kv8_plan_host.py"]
    r = subprocess.run(cmd, capture_output=True, text=True, env=env, cwd=ROOT, timeout=900)
    out = r.stdout + r.stderr
    if "ASan runtime does not come first" in out:
        pytest.skip("another preloaded library precedes the sanitizer runtime in this environment")
    assert r.returncode == 0, out[-4000:]
    assert "passed" in r.stdout and "failed" not in r.stdout and "AddressSanitizer" not in out and "runtime error" not in out, out[-4000:]
