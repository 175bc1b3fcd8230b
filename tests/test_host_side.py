"""What the host sides of the C ABI share, compiled alone against stand-ins of the CUDA calls it makes."""
import os
import shutil
import subprocess

import pytest

from paper_2609_03079_b200 import build

PROGRAM = r"""
#include "ls_host.cuh"
#include <cstdlib>
#include <new>

static bool g_no_memory = false;
static int g_events = 0;
void* operator new(std::size_t n) {
  if (g_no_memory) throw std::bad_alloc();
  return std::malloc(n ? n : 1);
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }
static int g_create_left = 1000;
extern "C" cudaError_t cudaEventCreate(cudaEvent_t* e) {
  if (g_create_left-- <= 0) return cudaErrorMemoryAllocation;
  *e = reinterpret_cast<cudaEvent_t>(++g_events);
  return cudaSuccess;
}
extern "C" cudaError_t cudaEventRecord(cudaEvent_t, cudaStream_t) { return cudaSuccess; }
extern "C" cudaError_t cudaEventDestroy(cudaEvent_t) { --g_events; return cudaSuccess; }

int main() {
  ls_host::g_timing = 1;
  { ls_host::KernelTimer t(5, nullptr); }
  if (ls_host::g_timed.size() != 1 || g_events != 2) return 1;
  ls_host::g_timed.shrink_to_fit();
  g_no_memory = true;
  { ls_host::KernelTimer t(5, nullptr); }  // there is no room to note it
  g_no_memory = false;
  if (ls_host::g_timed.size() != 1 || g_events != 2) return 2;
  g_create_left = 1;
  { ls_host::KernelTimer t(5, nullptr); }  // its second event cannot be made
  return ls_host::g_timed.size() == 1 && g_events == 2 ? 0 : 3;
}
"""


def test_a_timed_launch_that_cannot_be_noted_throws_nothing_and_keeps_nothing(tmp_path):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    src, exe = tmp_path / "timer.cpp", tmp_path / "timer"
    src.write_text(PROGRAM)
    cuda = os.path.join(os.path.dirname(os.path.dirname(build._nvcc())), "include")
    res = subprocess.run(["g++", "-std=c++17", "-O1", "-I", build.CSRC, "-I", cuda, str(src), "-o", str(exe)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    assert subprocess.run([str(exe)], capture_output=True).returncode == 0
