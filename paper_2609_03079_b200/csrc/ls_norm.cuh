// The norms before and after a block fused with its gate, residual scale and residual sum, one row (token) at a time:
//   t = N(y) w_post (or y);  x' = x + scale * gate * t;  h = N(x') w_pre (or x'),  N(z) = z / sqrt(mean z^2 + eps).
// Sums of squares, x' and h are fp32; x' and h are rounded once, when they are stored (h is made from the unrounded x').
#pragma once
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
__device__ __forceinline__ float ld1(const void* p, long long i) {
  if (DT == DT_F32) return static_cast<const float*>(p)[i];
  return widen<DT == DT_F32 ? 0 : DT>(static_cast<const uint16_t*>(p)[i]);
}
template <int DT>
__device__ __forceinline__ void st1(void* p, long long i, float v) {
  if (DT == DT_F32) static_cast<float*>(p)[i] = v;
  else static_cast<uint16_t*>(p)[i] = narrow<DT == DT_F32 ? 0 : DT>(v);
}

// V elements from element i on (one 16- or two 32-byte loads where V is 8; the caller has checked the alignment).
template <int DT, int V>
__device__ __forceinline__ void ldv(const void* p, long long i, float (&f)[V]) {
  if constexpr (V == 1) f[0] = ld1<DT>(p, i);
  else if constexpr (DT == DT_F32) {
    const float4 a = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i), b = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i + 4);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  } else unpack8<DT>(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i), f);
}
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

// A row is held in registers, K chunks of V elements per thread, so that everything is read once and all loads are under way
// before the first sum; a row belongs to a block, or (WARP) to one of its warps.
template <int XT, int BT, int V, int K, bool WARP>
__global__ void __launch_bounds__(WARP ? 256 : 1024) ls_norm_kernel(const NormArgs A) {
  __shared__ float s_sum[2][32];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const long long t = WARP ? (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
  const int tid = WARP ? threadIdx.x & 31 : threadIdx.x, nt = WARP ? 32 : blockDim.x;
  if (WARP && t >= A.n) return;
  const int chunks = A.d / V;
  float x[K][V], y[K][V], g[K][V];
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const int c = tid + i * nt;
#pragma unroll
    for (int e = 0; e < V; ++e) { x[i][e] = 0.f; y[i][e] = 0.f; g[i][e] = 1.f; }
    if (c >= chunks) continue;
    ldv<XT, V>(A.x, t * A.x_stride + (long long)c * V, x[i]);
    if (A.y) ldv<BT, V>(A.y, t * A.y_stride + (long long)c * V, y[i]);
    if (A.gate) ldv<BT, V>(A.gate, t * A.gate_stride + (long long)c * V, g[i]);
  }
  if (A.y) {
    float f = A.scale;
    if (A.post) {
      float q = 0.f;
#pragma unroll
      for (int i = 0; i < K; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) q = fmaf(y[i][e], y[i][e], q);
      f *= 1.f / sqrtf(row_sum<WARP>(q, s_sum[0]) / A.d + A.eps);
    }
#pragma unroll
    for (int i = 0; i < K; ++i) {
      const int c = tid + i * nt;
      float w[V];
#pragma unroll
      for (int e = 0; e < V; ++e) w[e] = f;
      if (A.w_post && c < chunks) {
        ldv<DT_F32, V>(A.w_post, (long long)c * V, w);
#pragma unroll
        for (int e = 0; e < V; ++e) w[e] *= f;
      }
#pragma unroll
      for (int e = 0; e < V; ++e) x[i][e] += y[i][e] * w[e] * g[i][e];
    }
  }
  if (A.x_out) {
#pragma unroll
    for (int i = 0; i < K; ++i)
      if (tid + i * nt < chunks) stv<XT, V>(A.x_out, t * A.x_out_stride + (long long)(tid + i * nt) * V, x[i]);
  }
  if (!A.h) return;
  float r = 1.f;
  if (A.pre) {
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < K; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) q = fmaf(x[i][e], x[i][e], q);
    r = 1.f / sqrtf(row_sum<WARP>(q, s_sum[1]) / A.d + A.eps);
  }
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const int c = tid + i * nt;
    if (c >= chunks) continue;
    float w[V];
#pragma unroll
    for (int e = 0; e < V; ++e) w[e] = 1.f;
    if (A.w_pre) ldv<DT_F32, V>(A.w_pre, (long long)c * V, w);
#pragma unroll
    for (int e = 0; e < V; ++e) x[i][e] *= r * w[e];
    stv<BT, V>(A.h, t * A.h_stride + (long long)c * V, x[i]);
  }
}

}  // namespace ls
