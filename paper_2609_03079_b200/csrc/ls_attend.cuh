// Attention over a paged cache whose first positions may be shared by the whole batch.
//
// Row (token t of sequence b, query head h) attends the keys j of [lo, hi), hi = position + 1, lo = hi - window (or 0):
//   s_j = scale <q, k_j>;  out = sum e^(s_j - M) v_j / sum e^(s_j - M);  lse = M + ln sum e^(s_j - M);  nothing seen: 0, -inf.
// Any cut of the keys into parts joins exactly: with (o_c, lse_c) of each part, out = sum_c e^(lse_c - lse) o_c.
#pragma once
#include "ls_common.cuh"

namespace ls {

struct AttendArgs {
  const void* q;       // [n_seqs * q_len][heads][dim], token stride q_stride
  void* out;           // same shape, token stride out_stride
  float* lse;          // [n_seqs * q_len][heads] or NULL
  const void* k;       // pages; element (page, slot, head, i) at page * page_stride + slot * token_stride + head * head_stride + i
  const void* v;
  const int32_t* seq_len;
  const int32_t* table;         // [n_seqs][table_stride], table_width entries of each row are valid
  const int32_t* prefix_pages;  // pages of the positions [0, prefix)
  int* status;
  float* part_o;       // parts of rows: normalised outputs and
  float* part_lse;     // their lse in units of log 2
  int64_t q_stride, out_stride, page_stride, token_stride, head_stride, table_stride;
  int32_t n_seqs, q_len, heads, kv_heads, group, dim;
  int32_t page, n_pages, table_width, prefix, window;
  int32_t splits;
  float scale_log2;    // softmax scale * log2(e)
};

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two fp32 values in a register pair, and arithmetic on both halves at once.
__device__ __forceinline__ uint64_t pair32(uint32_t lo, uint32_t hi) { return (uint64_t)hi << 32 | lo; }
__device__ __forceinline__ uint64_t both(float x) { return pair32(__float_as_uint(x), __float_as_uint(x)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float lo32(uint64_t x) { return __uint_as_float((uint32_t)x); }
__device__ __forceinline__ float hi32(uint64_t x) { return __uint_as_float((uint32_t)(x >> 32)); }
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

template <int WD>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if (WD == WD_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

template <int WD>
__device__ __forceinline__ uint16_t narrow16(float x) {
  uint16_t r;
  if (WD == WD_BF16) asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(r) : "f"(x));
  else asm("cvt.rn.f16.f32 %0, %1;" : "=h"(r) : "f"(x));
  return r;
}

template <int WD>
__device__ __forceinline__ void load8(const uint16_t* p, bool vec, float (&f)[8]) {
  uint4 v;
  if (vec) v = ldg128(p);
  else {
    v.x = p[0] | (uint32_t)p[1] << 16; v.y = p[2] | (uint32_t)p[3] << 16;
    v.z = p[4] | (uint32_t)p[5] << 16; v.w = p[6] | (uint32_t)p[7] << 16;
  }
  unpack8<WD>(v, f);
}

// Positions that the kernels count in 32 bits: what they add to one (tiles, batches of page numbers) stays below 2^31.
constexpr int MAX_POSITIONS = 0x7fff0000;

// Length of a sequence as far as its table and the positions reach; a longer or negative one is reported.
__device__ __forceinline__ int attend_len(const AttendArgs& A, int b, bool report) {
  const int n = A.seq_len[b];
  const long long most = min((long long)A.table_width * A.page, (long long)MAX_POSITIONS);
  if (n < 0 || n > most) {
    if (report) set_status(A.status, ST_BAD_INDEX);
    return n < 0 ? 0 : (int)most;
  }
  return n;
}

// ---- one block per (token, key head, up to NG of its query heads, split of the keys) --------------------------------------
// The route for every layout: any page size, any head dimension that is a multiple of 8 up to 256, any element alignment (what the
// tile kernel cannot copy as boxes).  Bound by its own instructions, a fused multiply-add per component, row and key: 64 / 8 heads
// over 100001 keys 1027 us (400 GB/s) where the tile kernel takes 71; a shared prefix is read again for every sequence.
// A key belongs to LPK lanes (8 components each), a warp reads 32 / LPK keys at a time and its lane groups and the four
// warps hold running (maximum, sum, output) triples that are joined once at the end.  All of it in fp32.
constexpr int AR_THREADS = 128;

template <int WD, int NG>
__global__ void __launch_bounds__(AR_THREADS) ls_attend_rows_kernel(const AttendArgs A, int lpk, int vec) {
  extern __shared__ float s_row[];  // [4 warps][NG][dim + 2]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int gt = (A.group + NG - 1) / NG;
  long long x = blockIdx.x;
  const int split = (int)(x % A.splits); x /= A.splits;
  const int g0 = (int)(x % gt) * NG; x /= gt;
  const int h = (int)(x % A.kv_heads);
  const long long t = x / A.kv_heads;
  const int b = (int)(t / A.q_len), i = (int)(t % A.q_len);
  const int len = attend_len(A, b, tid == 0 && split == 0);
  const int hi = max(len - A.q_len + i + 1, 0);
  const int lo = A.window > 0 ? max(hi - A.window, 0) : 0;
  const int n = hi - lo;
  const int a0 = lo + (int)((long long)n * split / A.splits), a1 = lo + (int)((long long)n * (split + 1) / A.splits);
  const int chunk = lane % lpk, sub = lane / lpk, kpw = 32 / lpk;
  const bool live = chunk * 8 < A.dim;
  const int ng = min(NG, A.group - g0);

  float q[NG][8], acc[NG][8], m[NG], l[NG];
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    m[g] = -INFINITY; l[g] = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) { q[g][e] = 0.f; acc[g][e] = 0.f; }
    if (live && g < ng) {
      load8<WD>(static_cast<const uint16_t*>(A.q) + t * A.q_stride + (long long)(h * A.group + g0 + g) * A.dim + chunk * 8, vec & 2, q[g]);
    }
  }
  const int32_t* row_table = A.table + (long long)b * A.table_stride;
  for (int base = a0 + warp * kpw; base < a1; base += 4 * kpw) {
    const int key = base + sub;
    bool on = key < a1;
    float kf[8], vf[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { kf[e] = 0.f; vf[e] = 0.f; }
    if (on) {
      const int pg = key / A.page, slot = key - pg * A.page;
      const int id = key < A.prefix ? A.prefix_pages[pg] : row_table[pg];
      if (id < 0 || id >= A.n_pages) {  // the key is left out
        set_status(A.status, ST_BAD_INDEX);
        on = false;
      } else if (live) {
        const long long off = id * A.page_stride + slot * A.token_stride + h * A.head_stride + chunk * 8;
        load8<WD>(static_cast<const uint16_t*>(A.k) + off, vec & 1, kf);
        load8<WD>(static_cast<const uint16_t*>(A.v) + off, vec & 1, vf);
      }
    }
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(q[g][e], kf[e], s);
      for (int o = lpk >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      s *= A.scale_log2;
      if (on) {
        if (s > m[g]) {
          const float f = ex2(m[g] - s);
          m[g] = s;
          l[g] *= f;
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[g][e] *= f;
        }
        // (a score of -inf under a maximum of -inf weighs nothing; a NaN score makes the row NaN)
        const float p = s == -INFINITY ? 0.f : ex2(s - m[g]);
        l[g] += p;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[g][e] = fmaf(p, vf[e], acc[g][e]);
      }
    }
  }
  // join the lane groups of a warp, then the warps
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    for (int o = lpk; o < 32; o <<= 1) {
      const float m2 = __shfl_xor_sync(0xffffffffu, m[g], o), l2 = __shfl_xor_sync(0xffffffffu, l[g], o);
      const float mm = fmaxf(m[g], m2);
      const float f1 = m[g] == -INFINITY ? 0.f : ex2(m[g] - mm), f2 = m2 == -INFINITY ? 0.f : ex2(m2 - mm);
      l[g] = l[g] * f1 + l2 * f2;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float a2 = __shfl_xor_sync(0xffffffffu, acc[g][e], o);
        acc[g][e] = acc[g][e] * f1 + a2 * f2;
      }
      m[g] = mm;
    }
    if (sub == 0 && live) {
      float* r = s_row + (warp * NG + g) * (A.dim + 2);
#pragma unroll
      for (int e = 0; e < 8; ++e) r[chunk * 8 + e] = acc[g][e];
      if (chunk == 0) { r[A.dim] = m[g]; r[A.dim + 1] = l[g]; }
    }
  }
  __syncthreads();
  for (int j = tid; j < ng * A.dim; j += AR_THREADS) {
    const int g = j / A.dim, c = j - g * A.dim;
    float mm = -INFINITY, ll = 0.f, o = 0.f;
    for (int w = 0; w < 4; ++w) mm = fmaxf(mm, s_row[(w * NG + g) * (A.dim + 2) + A.dim]);
    for (int w = 0; w < 4; ++w) {
      const float* r = s_row + (w * NG + g) * (A.dim + 2);
      const float f = r[A.dim] == -INFINITY ? 0.f : ex2(r[A.dim] - mm);
      ll += f * r[A.dim + 1];
      o += f * r[c];
    }
    const float res = ll == 0.f ? 0.f : o / ll;
    const float lse2 = ll == 0.f ? -INFINITY : mm + log2f(ll);
    const long long row = t * A.heads + h * A.group + g0 + g;
    if (A.splits == 1) {
      static_cast<uint16_t*>(A.out)[t * A.out_stride + (long long)(h * A.group + g0 + g) * A.dim + c] = (uint16_t)pack2<WD>(res, 0.f);
      if (c == 0 && A.lse) A.lse[row] = lse2 * LN2;
    } else {
      const long long pr = (long long)split * A.n_seqs * A.q_len * A.heads + row;
      A.part_o[pr * A.dim + c] = res;
      if (c == 0) A.part_lse[pr] = lse2;
    }
  }
}

// ---- joins the splits of the kernel above: one warp per row, in split order ------------------------------------------------
template <int WD>
__global__ void __launch_bounds__(256) ls_attend_rows_join_kernel(const AttendArgs A) {
  const long long rows = (long long)A.n_seqs * A.q_len * A.heads;
  const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (row >= rows) return;
  float mm = -INFINITY;
  for (int s = 0; s < A.splits; ++s) mm = fmaxf(mm, A.part_lse[s * rows + row]);
  float tot = 0.f;
  for (int s = 0; s < A.splits; ++s) {
    const float e = A.part_lse[s * rows + row];
    tot += e == -INFINITY ? 0.f : ex2(e - mm);
  }
  const long long t = row / A.heads;
  const int h = (int)(row - t * A.heads);
  const float inv = tot == 0.f ? 0.f : 1.f / tot;
  for (int c = lane; c < A.dim; c += 32) {
    float o = 0.f;
    for (int s = 0; s < A.splits; ++s) {
      const float e = A.part_lse[s * rows + row];
      if (e != -INFINITY) o = fmaf(ex2(e - mm) * inv, A.part_o[(s * rows + row) * A.dim + c], o);
    }
    static_cast<uint16_t*>(A.out)[t * A.out_stride + (long long)h * A.dim + c] = (uint16_t)pack2<WD>(o, 0.f);
  }
  if (lane == 0 && A.lse) A.lse[row] = tot == 0.f ? -INFINITY : (mm + log2f(tot)) * LN2;
}

}  // namespace ls
