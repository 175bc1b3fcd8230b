// The norms before and after a block fused with its gate, residual scale and residual sum, one row (token) at a time:
//   t = N(y) w_post (or y);  x' = x + scale * gate * t;  h = N(x') w_pre (or x'),  N(z) = z / sqrt(mean z^2 + eps).
// Sums of squares, x' and h are fp32; x' and h are rounded once, when they are stored (h is made from the unrounded x').
#pragma once
#include <type_traits>

#include "ls_append.cuh"
#include "ls_attend.cuh"
#include "ls_common.cuh"

namespace ls {

constexpr int DT_F32 = 2;  // beside WD_BF16 and WD_FP16

struct NormArgs {
  const void* x;        // [n][d] residual
  const void* y;        // [n][d] output of the block, or NULL (x' = x)
  void* x_out;          // NULL: not wanted; may be x
  void* h;              // NULL: not wanted; may be y
  const float* w_post;  // [d] or NULL
  const float* w_pre;   // [d] or NULL
  const void* gate;     // [d] (gate_stride 0) or [n][d], of y's type, or NULL
  int64_t x_stride, y_stride, x_out_stride, h_stride, gate_stride;
  int32_t n, d, post, pre;
  float scale, eps;
};

template <int DT>
__device__ __forceinline__ void st1(void* p, long long i, float v) {
  if (DT == DT_F32) static_cast<float*>(p)[i] = v;
  else static_cast<uint16_t*>(p)[i] = narrow<DT == DT_F32 ? 0 : DT>(v);
}

// V elements as they lie in memory (one 16-byte load, or two of them, where V is 8; the caller has checked the alignment).
template <int DT, int V>
struct Chunk {
  using Word = std::conditional_t<DT == DT_F32, float, uint16_t>;
  static constexpr int N = V == 1 ? 1 : DT == DT_F32 ? 2 : 1;
  std::conditional_t<V == 1, Word, uint4> r[N];
  __device__ __forceinline__ void load(const void* p, long long i) {
    const Word* q = static_cast<const Word*>(p) + i;
    if constexpr (V == 1) r[0] = *q;
    else {
#pragma unroll
      for (int k = 0; k < N; ++k) r[k] = reinterpret_cast<const uint4*>(q)[k];
    }
  }
  __device__ __forceinline__ void clear() {
    if constexpr (V == 1) r[0] = Word(0);
    else {
#pragma unroll
      for (int k = 0; k < N; ++k) r[k] = make_uint4(0u, 0u, 0u, 0u);
    }
  }
  __device__ __forceinline__ void get(float (&f)[V]) const {
    if constexpr (V == 1) {
      if constexpr (DT == DT_F32) f[0] = r[0];
      else f[0] = widen<DT>(r[0]);
    } else if constexpr (DT == DT_F32) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        f[4 * k] = __uint_as_float(r[k].x); f[4 * k + 1] = __uint_as_float(r[k].y);
        f[4 * k + 2] = __uint_as_float(r[k].z); f[4 * k + 3] = __uint_as_float(r[k].w);
      }
    } else unpack8<DT>(r[0], f);
  }
};
template <int DT, int V>
__device__ __forceinline__ void stv(void* p, long long i, const float (&f)[V]) {
  if constexpr (V == 1) st1<DT>(p, i, f[0]);
  else if constexpr (DT == DT_F32) {
    float4* d = reinterpret_cast<float4*>(static_cast<float*>(p) + i);
    d[0] = make_float4(f[0], f[1], f[2], f[3]);
    d[1] = make_float4(f[4], f[5], f[6], f[7]);
  } else
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + i) =
        make_uint4(pack2<DT>(f[0], f[1]), pack2<DT>(f[2], f[3]), pack2<DT>(f[4], f[5]), pack2<DT>(f[6], f[7]));
}

// Sum over a row's threads (a warp, or the block through `s`, a buffer used once per launch); every thread gets it.
template <bool WARP>
__device__ __forceinline__ float row_sum(float v, float* s) {
  v = warp_sum(v);
  if (WARP) return v;
  const int lane = threadIdx.x & 31, nw = blockDim.x >> 5;
  if (lane == 0) s[threadIdx.x >> 5] = v;
  __syncthreads();
  return warp_sum(lane < nw ? s[lane] : 0.f);
}

// A row is held in registers, K chunks of V elements per thread, as it lies in memory until it is used, so that everything is
// read once, all loads are under way before the first sum, and two blocks of 512 threads fit an SM (64 registers a thread).  A
// row belongs to a block, or (WARP) to one of its warps.  Gains are asked for ahead of the sum before their use where that
// takes few registers (one chunk a thread: few rows, where latency counts), else when they are used (they are in L1 then).
// Bound by memory for many rows: 8192 x 8192 in bf16 with a gate, 671 MB, 120 to 126 us, 5.3 to 5.6 TB/s, 0.82 to 0.87 of measured; 8192 x 4096 with the
// residual in fp32 66 us, 6.1 TB/s.  One row of 4096: 3 us a call, 2.1 on the device (two sums over the block).  Widths that are
// no multiple of 8 go one element at a time: 200 x 5121 8.6 us against 5.8 for 200 x 5120.
template <int XT, int BT, int V, int K, bool WARP>
__global__ void __launch_bounds__(WARP ? 256 : 1024) ls_norm_kernel(const NormArgs A) {
  constexpr bool AHEAD = V * K <= 8;
  __shared__ float s_sum[2][32];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const long long t = WARP ? (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
  const int tid = WARP ? threadIdx.x & 31 : threadIdx.x, nt = WARP ? 32 : blockDim.x;
  if (WARP && t >= A.n) return;
  const int chunks = A.d / V;
  const bool has_y = A.y != nullptr, has_g = A.gate != nullptr;
  Chunk<XT, V> xr[K];
  Chunk<BT, V> yr[K], gr[K];
  Chunk<DT_F32, V> w1[AHEAD ? K : 1], w2[AHEAD ? K : 1];
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const int c = (tid + i * nt) * V;
    xr[i].clear(); yr[i].clear(); gr[i].clear();
    if (tid + i * nt >= chunks) continue;
    xr[i].load(A.x, t * A.x_stride + c);
    if (has_y) yr[i].load(A.y, t * A.y_stride + c);
    if (has_g) gr[i].load(A.gate, t * A.gate_stride + c);
    if (AHEAD && A.w_post) w1[i].load(A.w_post, c);
    if (AHEAD && A.w_pre) w2[i].load(A.w_pre, c);
  }
  float f = A.scale;
  if (has_y && A.post) {
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < K; ++i) {
      float y[V];
      yr[i].get(y);
#pragma unroll
      for (int e = 0; e < V; ++e) q = fmaf(y[e], y[e], q);
    }
    f *= 1.f / sqrtf(row_sum<WARP>(q, s_sum[0]) / A.d + A.eps);
  }
  float x[K][V], q = 0.f;
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const int c = (tid + i * nt) * V;
    const bool on = tid + i * nt < chunks;
    xr[i].get(x[i]);
    if (has_y) {
      float y[V], m[V];
      yr[i].get(y);
#pragma unroll
      for (int e = 0; e < V; ++e) y[e] *= f;
      if (A.w_post && on) {
        if (!AHEAD) w1[0].load(A.w_post, c);
        w1[AHEAD ? i : 0].get(m);
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] *= m[e];
      }
      if (has_g) {
        gr[i].get(m);
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] *= m[e];
      }
#pragma unroll
      for (int e = 0; e < V; ++e) x[i][e] += y[e];
    }
    if (A.x_out && on) stv<XT, V>(A.x_out, t * A.x_out_stride + c, x[i]);
#pragma unroll
    for (int e = 0; e < V; ++e) q = fmaf(x[i][e], x[i][e], q);
  }
  if (!A.h) return;
  const float r = A.pre ? 1.f / sqrtf(row_sum<WARP>(q, s_sum[1]) / A.d + A.eps) : 1.f;
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const int c = (tid + i * nt) * V;
    if (tid + i * nt >= chunks) continue;
#pragma unroll
    for (int e = 0; e < V; ++e) x[i][e] *= r;
    if (A.w_pre) {
      float m[V];
      if (!AHEAD) w2[0].load(A.w_pre, c);
      w2[AHEAD ? i : 0].get(m);
#pragma unroll
      for (int e = 0; e < V; ++e) x[i][e] *= m[e];
    }
    stv<BT, V>(A.h, t * A.h_stride + c, x[i]);
  }
}

}  // namespace ls
