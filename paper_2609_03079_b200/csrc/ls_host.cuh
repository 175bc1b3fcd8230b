// What the host sides of the C ABI share: the calling thread's error text, launch accounting, optional kernel timing, the
// device guard and checked allocation.
#pragma once
#include "../../include/leanstream.h"

#include <cuda_runtime.h>

#include <atomic>
#include <cstdarg>
#include <cstdio>
#include <mutex>
#include <string>
#include <utility>
#include <vector>

namespace ls_host {

inline thread_local std::string g_err;
inline std::atomic<int64_t> g_launches{0};

inline int32_t fail(int32_t code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  try { g_err = buf; } catch (...) { g_err.clear(); }  // (a message too long for memory is lost, not thrown)
  return code;
}

#define LS_CUDA(call)                                                                         \
  do {                                                                                        \
    cudaError_t e_ = (call);                                                                  \
    if (e_ != cudaSuccess) return fail(LS_ERR_CUDA, "%s: %s", #call, cudaGetErrorString(e_)); \
  } while (0)

#define LS_LAUNCHED()                                                                                   \
  do {                                                                                                  \
    g_launches.fetch_add(1, std::memory_order_relaxed);                                                 \
    cudaError_t e_ = cudaPeekAtLastError();                                                             \
    if (e_ != cudaSuccess) return fail(LS_ERR_CUDA, "kernel launch (%s:%d): %s", __FILE__, __LINE__,    \
                                       cudaGetErrorString(e_));                                        \
  } while (0)

// Optional per-kernel timing with CUDA events on the launching stream (roofline accounting; off by default).
struct TimedLaunch { int kind; cudaEvent_t a, b; };
inline std::atomic<int> g_timing{0};
inline std::mutex g_timing_mu;
inline std::vector<TimedLaunch> g_timed;

struct KernelTimer {
  cudaStream_t st;
  TimedLaunch t{};
  bool on;
  KernelTimer(int kind, cudaStream_t s) : st(s), on(g_timing.load(std::memory_order_relaxed) != 0) {
    if (!on) return;
    t.kind = kind;
    if (cudaEventCreate(&t.a) != cudaSuccess) { on = false; return; }
    if (cudaEventCreate(&t.b) != cudaSuccess) { cudaEventDestroy(t.a); on = false; return; }
    cudaEventRecord(t.a, st);
  }
  ~KernelTimer() {
    if (!on) return;
    cudaEventRecord(t.b, st);
    try {
      std::lock_guard<std::mutex> lk(g_timing_mu);
      g_timed.push_back(t);
    } catch (...) {  // (no memory for it: the launch goes untimed, nothing is thrown through the C ABI)
      cudaEventDestroy(t.a);
      cudaEventDestroy(t.b);
    }
  }
};

struct DeviceGuard {
  int prev = -1;
  explicit DeviceGuard(int dev) {
    cudaGetDevice(&prev);
    if (prev != dev) cudaSetDevice(dev);
  }
  ~DeviceGuard() {
    int cur = -1;
    cudaGetDevice(&cur);
    if (prev >= 0 && cur != prev) cudaSetDevice(prev);
  }
};

template <typename T>
int32_t dalloc(T** p, size_t n) {
  *p = nullptr;
  if (n == 0) n = 1;
  cudaError_t e = cudaMalloc(reinterpret_cast<void**>(p), n * sizeof(T));
  if (e != cudaSuccess) return fail(e == cudaErrorMemoryAllocation ? LS_ERR_NOMEM : LS_ERR_CUDA, "cudaMalloc(%zu bytes): %s",
                                    n * sizeof(T), cudaGetErrorString(e));
  return LS_OK;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Each pointer (NULL among them) lies at a multiple of its element's `size` bytes: the kernels' accesses would fault otherwise.
template <class... P>
bool elements_aligned(size_t size, P... p) {
  return ((reinterpret_cast<uintptr_t>(p) | ...) & (size - 1)) == 0;
}

// Launches that may start while the kernel in front of them ends; the kernels wait for it before they touch memory.
template <class... P, class... Q>
int32_t launch_early(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, Q&&... args) {
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  LS_CUDA(cudaLaunchKernelEx(&cfg, kernel, std::forward<Q>(args)...));
  LS_LAUNCHED();
  return LS_OK;
}

#define LS_TRY(expr)              \
  do {                            \
    int32_t rc_ = (expr);         \
    if (rc_ != LS_OK) return rc_; \
  } while (0)

}  // namespace ls_host
