// Keys and values of new tokens go into their slots of a paged cache, queries and keys turned by their positions on the way.
//
// The first `rope_dim` components of a head are turned in pairs (x1, x2) -> (x1 c - x2 s, x2 c + x1 s), c and s from row
// `position` of a table the caller keeps ([positions][rope_dim]: rope_dim / 2 cosines, then as many sines); a pair is
// (i, i + rope_dim / 2), or (2 i, 2 i + 1) when interleaved.  The arithmetic is fp32, rounded once to the 16-bit type.
#pragma once
#include "ls_attend.cuh"
#include "ls_common.cuh"

namespace ls {

struct AppendArgs {
  const uint16_t* q;   // [n_tokens][heads][dim] at token stride q_stride, or NULL
  uint16_t* q_out;
  const uint16_t* k;   // [n_tokens][kv_heads][dim]
  const uint16_t* v;
  uint16_t* k_pages;
  uint16_t* v_pages;
  const int32_t* seq;
  const int32_t* pos;
  const int32_t* table;
  const float* rope;
  int* status;
  int64_t q_stride, q_out_stride, k_stride, v_stride, page_stride, token_stride, head_stride, table_stride;
  int32_t n_tokens, n_seqs, heads, kv_heads, dim, page, n_pages, table_width, rope_dim, rope_positions, interleaved;
};

template <int WD>
__device__ __forceinline__ float widen(uint16_t x) {
  if (WD == WD_BF16) return __uint_as_float((uint32_t)x << 16);
  return __half2float(__ushort_as_half(x));
}
template <int WD>
__device__ __forceinline__ uint16_t narrow(float x) {
  uint16_t r;
  if (WD == WD_BF16) asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(r) : "f"(x));
  else asm("cvt.rn.f16.f32 %0, %1;" : "=h"(r) : "f"(x));
  return r;
}

// Where token t's keys and values go (element offset of head 0 in the pages), or -1: padding (a negative sequence or
// position) is passed over silently, anything out of range is passed over and reported.  (What becomes of the token's query does
// not depend on this: it is turned if its position is in the rotation table.)
__device__ __forceinline__ long long append_slot(const AppendArgs& A, int sq, int ps) {
  if (sq < 0 || ps < 0) return -1;
  const int pg = ps / A.page;
  if (sq >= A.n_seqs || pg >= A.table_width || (A.rope_dim > 0 && ps >= A.rope_positions)) { set_status(A.status, ST_BAD_INDEX); return -1; }
  const int id = A.table[(long long)sq * A.table_stride + pg];
  if (id < 0 || id >= A.n_pages) { set_status(A.status, ST_BAD_INDEX); return -1; }
  return id * A.page_stride + (long long)(ps - pg * A.page) * A.token_stride;
}

// A block of one token, or (SEVERAL) of as many as fit with `width` threads each; 16-byte loads and stores.  A thread has the
// same two chunks of eight components in every head that it visits (chunks whose components are each other's partners, or two
// neighbours where nothing is turned), so that it reads its cosines and sines once per token.  For head and rotation sizes of a
// multiple of 16 and 16-byte aligned operands.
// Bound by memory: 16 x 1023 tokens of 64 + 2 x 8 heads of 128, 679 MB, 119 us, 5.7 TB/s, 0.88 of measured (the pair kernel below:
// 579 us; with the token's place looked up before the first loads instead of behind them: 137).  One token: 2.9 us a call,
// three dependent reads (place, page, slot) and the launch.
template <int WD, bool SEVERAL>
__global__ void __launch_bounds__(256) ls_append_kernel(const AppendArgs A, int width) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int mine = SEVERAL ? threadIdx.x / width : 0, tid = SEVERAL ? threadIdx.x - mine * width : threadIdx.x;
  const long long t = SEVERAL ? (long long)blockIdx.x * (blockDim.x / width) + mine : blockIdx.x;
  const int per = A.dim / 16, nq = A.q ? A.heads : 0, heads = nq + 2 * A.kv_heads;
  const int i = tid % per, step = (SEVERAL ? width : (int)blockDim.x) / per;
  const bool turned = 16 * i < A.rope_dim;
  const int c0 = turned && !A.interleaved ? 8 * i : 16 * i, c1 = turned && !A.interleaved ? c0 + A.rope_dim / 2 : c0 + 8;
  if (tid >= step * per || (SEVERAL && (mine >= blockDim.x / width || t >= A.n_tokens))) return;
  auto source = [&](int hd) {
    return (hd < nq ? A.q + t * A.q_stride + (long long)hd * A.dim
            : hd < nq + A.kv_heads ? A.k + t * A.k_stride + (long long)(hd - nq) * A.dim
                                   : A.v + t * A.v_stride + (long long)(hd - nq - A.kv_heads) * A.dim);
  };
  // Two heads at a time; the first two are under way before the token's place and angles are looked up.
  uint4 a0, b0, a1, b1;
  auto fetch = [&](int hd) {
    const uint16_t *p = source(min(hd, heads - 1)), *q = source(min(hd + step, heads - 1));
    a0 = ld_stream128(p + c0); b0 = ld_stream128(p + c1);
    a1 = ld_stream128(q + c0); b1 = ld_stream128(q + c1);
  };
  int hd = tid / per;
  fetch(hd);
  const int sq = A.seq[t], ps = A.pos[t];
  float c[8], s[8];
  const bool in_table = ps >= 0 && ps < A.rope_positions;
  if (turned && in_table) {
    const float4* tab = reinterpret_cast<const float4*>(A.rope + (long long)ps * A.rope_dim + 8 * i);
    const float4* tas = reinterpret_cast<const float4*>(A.rope + (long long)ps * A.rope_dim + A.rope_dim / 2 + 8 * i);
    const float4 a = __ldg(tab), b = __ldg(tab + 1), e = __ldg(tas), f = __ldg(tas + 1);
    c[0] = a.x; c[1] = a.y; c[2] = a.z; c[3] = a.w; c[4] = b.x; c[5] = b.y; c[6] = b.z; c[7] = b.w;
    s[0] = e.x; s[1] = e.y; s[2] = e.z; s[3] = e.w; s[4] = f.x; s[5] = f.y; s[6] = f.z; s[7] = f.w;
  }
  const long long slot = append_slot(A, sq, ps);
  auto finish = [&](int hd, uint4 ra, uint4 rb) {
    uint16_t* dst;
    if (hd < nq) dst = A.q_out + t * A.q_out_stride + (long long)hd * A.dim;
    else if (slot < 0) return;
    else dst = hd < nq + A.kv_heads ? A.k_pages + slot + (hd - nq) * A.head_stride : A.v_pages + slot + (hd - nq - A.kv_heads) * A.head_stride;
    if (turned && in_table && hd < nq + A.kv_heads) {
      float a[8], b[8], x[8], y[8];
      unpack8<WD>(ra, a);
      unpack8<WD>(rb, b);
      if (A.interleaved) {  // pairs side by side: four in each chunk
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[2 * e] = a[2 * e] * c[e] - a[2 * e + 1] * s[e];
          x[2 * e + 1] = a[2 * e + 1] * c[e] + a[2 * e] * s[e];
          y[2 * e] = b[2 * e] * c[4 + e] - b[2 * e + 1] * s[4 + e];
          y[2 * e + 1] = b[2 * e + 1] * c[4 + e] + b[2 * e] * s[4 + e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) { x[e] = a[e] * c[e] - b[e] * s[e]; y[e] = b[e] * c[e] + a[e] * s[e]; }
      }
      ra = make_uint4(pack2<WD>(x[0], x[1]), pack2<WD>(x[2], x[3]), pack2<WD>(x[4], x[5]), pack2<WD>(x[6], x[7]));
      rb = make_uint4(pack2<WD>(y[0], y[1]), pack2<WD>(y[2], y[3]), pack2<WD>(y[4], y[5]), pack2<WD>(y[6], y[7]));
    }
    *reinterpret_cast<uint4*>(dst + c0) = ra;
    *reinterpret_cast<uint4*>(dst + c1) = rb;
  };
  for (;;) {
    if (hd < heads) finish(hd, a0, b0);
    if (hd + step < heads) finish(hd + step, a1, b1);
    hd += 2 * step;
    if (hd >= heads) break;
    fetch(hd);
  }
}

// One thread per pair of components: the route for any alignment and any even rope_dim.
template <int WD>
__global__ void __launch_bounds__(256) ls_append_pairs_kernel(const AppendArgs A) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const long long t = blockIdx.x;
  const int sq = A.seq[t], ps = A.pos[t];
  const long long slot = append_slot(A, sq, ps);
  const bool in_table = A.rope_dim == 0 || (ps >= 0 && ps < A.rope_positions);
  const int half = A.dim / 2, r2 = A.rope_dim / 2, nq = A.q ? A.heads : 0;
  const float* tab = A.rope + (long long)ps * A.rope_dim;
  for (int j = blockIdx.y * blockDim.x + threadIdx.x; j < (nq + 2 * A.kv_heads) * half; j += gridDim.y * blockDim.x) {
    const int hd = j / half, i = j - hd * half;
    const uint16_t* src;
    uint16_t* dst;
    bool turn = i < r2;
    if (hd < nq) {
      src = A.q + t * A.q_stride + (long long)hd * A.dim;
      dst = A.q_out + t * A.q_out_stride + (long long)hd * A.dim;
      turn = turn && in_table;
    } else {
      if (slot < 0) continue;
      const bool key = hd < nq + A.kv_heads;
      const int h = hd - nq - (key ? 0 : A.kv_heads);
      src = (key ? A.k + t * A.k_stride : A.v + t * A.v_stride) + (long long)h * A.dim;
      dst = (key ? A.k_pages : A.v_pages) + slot + h * A.head_stride;
      turn = turn && key;
    }
    // components of pair i: the turned ones first, the rest side by side
    int c0, c1;
    if (i < r2) { c0 = A.interleaved ? 2 * i : i; c1 = A.interleaved ? c0 + 1 : i + r2; }
    else { c0 = 2 * i; c1 = c0 + 1; }
    if (turn) {
      const float x1 = widen<WD>(src[c0]), x2 = widen<WD>(src[c1]), c = tab[i], s = tab[r2 + i];
      dst[c0] = narrow<WD>(x1 * c - x2 * s);
      dst[c1] = narrow<WD>(x2 * c + x1 * s);
    } else {
      const uint16_t a = src[c0], b = src[c1];
      dst[c0] = a;
      dst[c1] = b;
    }
  }
}

}  // namespace ls
