"""The library's error path on its own: host code alone, compiled here (no GPU)."""
import os
import shutil
import subprocess

import pytest

PKG = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                   "paper_2011_13824_amd")
PROGRAM = r"""
#include <cstdlib>
#include <new>
#include "host.hpp"
static bool none_left = false;
void* operator new(std::size_t n) {
  if (none_left) throw std::bad_alloc();
  return std::malloc(n);
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }
int main() {
  using namespace lirpa_host;
  if (fail(LIRPA_EINVAL, "width %d is outside [1, 2^20], as any message can be", 7) != LIRPA_EINVAL)
    return 1;
  if (g_err != "width 7 is outside [1, 2^20], as any message can be") return 2;
  none_left = true;
  int rc = 0;
  try {
    rc = fail(LIRPA_ENOMEM, "%0400d", 1);
  } catch (...) {
    return 3;
  }
  none_left = false;
  if (rc != LIRPA_ENOMEM || !g_err.empty()) return 4;
  return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"),
                    reason="needs g++ and the HIP headers")
def test_an_error_without_memory_for_its_message_is_still_one(tmp_path):
    src, exe = tmp_path / "errors.cpp", tmp_path / "errors"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + os.path.join(PKG, "csrc"),
                    "-I" + os.path.join(os.path.dirname(PKG), "include"), str(src), "-o", str(exe),
                    "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"],
                   check=True, capture_output=True, text=True)
    assert subprocess.run([str(exe)]).returncode == 0
