// The norms before and after a block fused with its gate, residual scale and residual sum, one row (token) at a time:
//   t = N(y) w_post (or y);  x' = x + scale * gate * t;  h = N(x') w_pre (or x'),  N(z) = z / sqrt(mean z^2 + eps).
// Sums of squares, x' and h are fp32; x' and h are rounded once, when they are stored (h is made from the unrounded x').
#pragma once
#include "ls_append.cuh"
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

// Sum over the block of one value per thread (every thread gets it); `s` has a word for each warp and one more.
__device__ __forceinline__ float block_sum(float v, float* s) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = (blockDim.x + 31) >> 5;
  v = warp_sum(v);
  __syncthreads();  // (the words may still be read from the sum before)
  if (lane == 0) s[warp] = v;
  __syncthreads();
  return warp_sum(lane < nw ? s[lane] : 0.f);
}

// One block per row, the row's x' kept in shared memory: the route for any width and alignment.
template <int XT, int BT>
__global__ void __launch_bounds__(512) ls_norm_rows_kernel(const NormArgs A) {
  extern __shared__ float s_x[];  // [d]
  __shared__ float s_sum[33];
  const long long t = blockIdx.x;
  const int tid = threadIdx.x, nt = blockDim.x;
  float f = A.scale;
  if (A.y && A.post) {
    float q = 0.f;
    for (int c = tid; c < A.d; c += nt) { const float y = ld1<BT>(A.y, t * A.y_stride + c); q = fmaf(y, y, q); }
    f *= 1.f / sqrtf(block_sum(q, s_sum) / A.d + A.eps);
  }
  float q = 0.f;
  for (int c = tid; c < A.d; c += nt) {
    float x = ld1<XT>(A.x, t * A.x_stride + c);
    if (A.y) {
      float z = ld1<BT>(A.y, t * A.y_stride + c) * f;
      if (A.w_post) z *= A.w_post[c];
      if (A.gate) z *= ld1<BT>(A.gate, t * A.gate_stride + c);
      x += z;
    }
    s_x[c] = x;
    if (A.x_out) st1<XT>(A.x_out, t * A.x_out_stride + c, x);
    q = fmaf(x, x, q);
  }
  if (!A.h) return;
  const float r = A.pre ? 1.f / sqrtf(block_sum(q, s_sum) / A.d + A.eps) : 1.f;
  for (int c = tid; c < A.d; c += nt) {
    float z = s_x[c] * r;
    if (A.w_pre) z *= A.w_pre[c];
    st1<BT>(A.h, t * A.h_stride + c, z);
  }
}

}  // namespace ls
