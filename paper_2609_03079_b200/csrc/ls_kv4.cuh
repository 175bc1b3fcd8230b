// A paged key/value cache held in 4 bits: where its parts lie, the append that quantises into it, the kernel that reads it back.
//
// `group` (32, 64 or 128) consecutive components of one token's key or value of one head share a scale and a zero of the cache's
// 16-bit type.  With x the components as a 16-bit cache would hold them (a key is turned in 64 bits, then rounded to 32 and to 16):
//   zero = min x;  scale = (max x - min x) / 15 in fp32, rounded to the type;  code = min(15, round((x - zero) / scale)), ties to even
// and scale * code + zero is what is held.  scale 0: all codes are 0.  A range that is not finite: scale and zero are NaN.
// Every step is one exactly rounded operation, so that codes do not depend on who computes them.
//
// A block (one page of one key head) is a row of tiles of 16 tokens, each contiguous so that one bulk copy brings it:
//   16 rows of key codes (dim / 2 bytes), 16 of value codes, 16 x (groups x (scale, zero)) of keys, the same of values.
// Inside a code row the words (eight codes, the lowest bits first) and the codes lie as the matrix instructions of the attention
// take them from shared memory, without bank conflicts (`key_word`, `value_word`).
#pragma once
#include "ls_append.cuh"
#include "ls_common.cuh"

namespace ls {

struct Kv4Pages {
  uint8_t* pages;        // block (page, head) at page * page_stride + head * head_stride
  const int32_t* table;
  int* status;
  int64_t page_stride, head_stride, table_stride;  // bytes, bytes, entries
  int32_t n_seqs, kv_heads, group, page, n_pages, table_width;
};

// Bytes of a tile of 16 tokens.
__host__ __device__ constexpr int kv4_tile(int dim, int group) { return 16 * (dim + 8 * (dim / group)); }

// Word of a key row that holds the components 8 w to 8 w + 7, in order.  The four threads that share a row in a matrix product take
// n words each with one load; rows of 128 bytes trade halves so that two neighbouring rows meet in different banks.
template <int D>
__host__ __device__ constexpr int key_word(int w, int row) {
  constexpr int n = D == 64 ? 2 : 4;
  const int turn = w / 4, half = (turn / n) ^ (D == 256 ? row & 1 : 0);
  return half * 4 * n + (w % 4) * n + turn % n;
}
// Word of a value row that holds the components 64 ws + 4 g ... + 3 in its low half and the ones 32 further in its high half.
// Pieces of 32 bytes trade places so that four rows meet in different banks.
template <int D>
__host__ __device__ constexpr int value_word(int g, int ws, int row) {
  constexpr int n = D / 64;
  const int at = g * n + ws;
  const int swap = D == 64 ? 0 : D == 128 ? (row >> 1) & 1 : row & 3;
  return ((at >> 3) ^ swap) * 8 + (at & 7);
}

// Byte offset in the pages of the tile of (sequence, position) for head 0, or -1: padding is passed over silently, anything out of
// range is passed over and reported.
__device__ __forceinline__ long long kv4_tile_at(const Kv4Pages& P, int sq, int ps, int limit, int tile_bytes, int& row) {
  if (sq < 0 || ps < 0) return -1;
  const int pg = ps / P.page, slot = ps - pg * P.page;
  row = slot & 15;
  if (sq >= P.n_seqs || pg >= P.table_width || ps >= limit) { set_status(P.status, ST_BAD_INDEX); return -1; }
  const int id = P.table[(long long)sq * P.table_stride + pg];
  if (id < 0 || id >= P.n_pages) { set_status(P.status, ST_BAD_INDEX); return -1; }
  return id * P.page_stride + (long long)(slot >> 4) * tile_bytes;
}

struct Kv4AppendArgs {
  Kv4Pages p;
  const uint16_t* q;   // [n_tokens][heads][dim] at token stride q_stride, or NULL
  uint16_t* q_out;
  const uint16_t* k;   // [n_tokens][kv_heads][dim]
  const uint16_t* v;
  const int32_t* seq;
  const int32_t* pos;
  const float* rope;
  int64_t q_stride, q_out_stride, k_stride, v_stride;
  int32_t n_tokens, heads, rope_dim, rope_positions, interleaved;
  int32_t kv_jobs, jobs;  // warps of a token: for its keys (and as many for its values), for all of it
  int32_t kv_vec, q_vec, rope_vec;
};

struct Quad { float x[4]; };

// Four consecutive components.
template <int WD>
__device__ __forceinline__ Quad load_quad(const uint16_t* p, bool vec) {
  uint2 r;
  if (vec) r = __ldg(reinterpret_cast<const uint2*>(p));
  else { r.x = p[0] | (uint32_t)p[1] << 16; r.y = p[2] | (uint32_t)p[3] << 16; }
  return {{widen<WD>((uint16_t)r.x), widen<WD>((uint16_t)(r.x >> 16)), widen<WD>((uint16_t)r.y), widen<WD>((uint16_t)(r.y >> 16))}};
}

// Quantises the lane's quad of a head (components 4 * quad ...) with the other lanes of its group, and stores it.
template <int WD, int D>
__device__ __forceinline__ void store_quad(const Kv4AppendArgs& A, const Quad& y, bool value, int quad, int row, uint8_t* tile) {
  const int lane = threadIdx.x & 31, span = A.p.group / 4;
  float lo = fminf(fminf(y.x[0], y.x[1]), fminf(y.x[2], y.x[3])), hi = -INFINITY;
#pragma unroll
  for (int e = 0; e < 4; ++e) hi = fmaxf(hi, y.x[e] != y.x[e] ? INFINITY : y.x[e]);  // (NaN must not get lost)
  for (int o = 1; o < span; o <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  const float range = hi - lo;
  const bool fine = range < INFINITY;
  const uint16_t scale16 = fine ? narrow<WD>(__fdiv_rn(range, 15.f)) : 0x7fff, zero16 = fine ? narrow<WD>(lo) : 0x7fff;
  const float scale = widen<WD>(scale16);
  uint32_t codes = 0;
  if (scale > 0.f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) codes |= (uint32_t)min(15, __float2int_rn(__fdiv_rn(y.x[e] - lo, scale))) << (4 * e);
  }
  // a word is two quads: neighbours of a key, 32 components apart of a value
  const uint32_t other = __shfl_xor_sync(0xffffffffu, codes, value ? 8 : 1);
  if (!tile) return;
  const bool low = value ? !(quad & 8) : !(quad & 1);
  const int word = value ? value_word<D>(quad & 7, quad >> 4, row) : key_word<D>(quad >> 1, row);
  if (low) *reinterpret_cast<uint32_t*>(tile + ((value ? 16 : 0) + row) * (D / 2) + 4 * word) = codes | other << 16;
  if (lane % span == 0) {
    const int groups = D / A.p.group;
    *reinterpret_cast<uint32_t*>(tile + 16 * D + (((value ? 16 : 0) + row) * groups + quad / span) * 4) = scale16 | (uint32_t)zero16 << 16;
  }
}

// The lane's quad of a key, turned by the token's row of the table (in 64 bits: the difference of two products rounds once there, so
// that the key and with it the codes do not depend on the order of operations), as the 16-bit type holds it.
template <int WD>
__device__ __forceinline__ Quad turned_quad(const Kv4AppendArgs& A, const Quad& a, const uint16_t* head, int d0, const float* tab) {
  const int r = A.rope_dim, r2 = r / 2;
  if (d0 >= r) return a;
  Quad b, c, s, y;
  if (A.rope_vec) {  // half of the turned part is a multiple of four: partners and angles are quads too
    const int j = A.interleaved ? d0 / 2 : d0 < r2 ? d0 : d0 - r2;
    if (A.interleaved) {
      const float2 c2 = __ldg(reinterpret_cast<const float2*>(tab + j)), s2 = __ldg(reinterpret_cast<const float2*>(tab + r2 + j));
      b = {{a.x[1], a.x[0], a.x[3], a.x[2]}}; c = {{c2.x, c2.x, c2.y, c2.y}}; s = {{s2.x, s2.x, s2.y, s2.y}};
    } else {
      const float4 c4 = __ldg(reinterpret_cast<const float4*>(tab + j)), s4 = __ldg(reinterpret_cast<const float4*>(tab + r2 + j));
      b = load_quad<WD>(head + (d0 < r2 ? d0 + r2 : d0 - r2), A.kv_vec);
      c = {{c4.x, c4.y, c4.z, c4.w}}; s = {{s4.x, s4.y, s4.z, s4.w}};
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int d = d0 + e;
      b.x[e] = c.x[e] = s.x[e] = 0.f;
      if (d >= r) continue;
      const int j = A.interleaved ? d / 2 : d < r2 ? d : d - r2;
      b.x[e] = widen<WD>(head[A.interleaved ? d ^ 1 : d < r2 ? d + r2 : d - r2]);
      c.x[e] = tab[j]; s.x[e] = tab[r2 + j];
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int d = d0 + e;
    if (d >= r) { y.x[e] = a.x[e]; continue; }
    const bool second = A.interleaved ? d & 1 : d >= r2;
    const double turn = (double)b.x[e] * (double)s.x[e];
    const double z = fma((double)a.x[e], (double)c.x[e], second ? turn : -turn);
    y.x[e] = widen<WD>(narrow<WD>(__double2float_rn(z)));
  }
  return y;
}

// A warp takes 1024 components of a token's queries, or 256 of its keys or of its values (two quads a lane, so that the lanes of a
// group sit side by side).  Queries are turned in fp32 and rounded once, as in the 16-bit append.
template <int WD, int D>
__global__ void __launch_bounds__(256) ls_kv4_append_kernel(const Kv4AppendArgs A) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int lane = threadIdx.x & 31;
  const unsigned long long id = (unsigned long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const long long t = (long long)(id / (unsigned)A.jobs);
  const int job = (int)(id - (unsigned long long)t * (unsigned)A.jobs);
  if (t >= A.n_tokens) return;
  if (job < 2 * A.kv_jobs) {
    const bool value = job >= A.kv_jobs;
    const int slab0 = 2 * (value ? job - A.kv_jobs : job);
    const uint16_t* token = value ? A.v + t * A.v_stride : A.k + t * A.k_stride;
    int head[2], quad[2];
    Quad a[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int slab = slab0 + i;  // 128 components
      head[i] = D == 64 ? slab * 2 + lane / 16 : D == 128 ? slab : slab / 2;
      quad[i] = D == 64 ? lane % 16 : D == 128 ? lane : lane + 32 * (slab & 1);
      a[i] = load_quad<WD>(token + (long long)min(head[i], A.p.kv_heads - 1) * D + 4 * quad[i], A.kv_vec);
    }
    const int sq = A.seq[t], ps = A.pos[t];
    int row = 0;
    const long long at = kv4_tile_at(A.p, sq, ps, A.rope_dim > 0 ? A.rope_positions : 0x7fffffff, kv4_tile(D, A.p.group), row);
    if (at < 0) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (!value && A.rope_dim > 0)
        a[i] = turned_quad<WD>(A, a[i], token + (long long)min(head[i], A.p.kv_heads - 1) * D, 4 * quad[i], A.rope + (long long)ps * A.rope_dim);
      store_quad<WD, D>(A, a[i], value, quad[i], row, head[i] < A.p.kv_heads ? A.p.pages + at + head[i] * A.p.head_stride : nullptr);
    }
    return;
  }
  const int ps = A.pos[t], r2 = A.rope_dim / 2;
  const bool turn = A.rope_dim > 0 && ps >= 0 && ps < A.rope_positions;
  const float* tab = A.rope + (long long)ps * A.rope_dim;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int item = (job - 2 * A.kv_jobs) * 64 + k * 32 + lane, hd = item / (D / 16), i = item % (D / 16);
    if (hd >= A.heads) return;
    const uint16_t* src = A.q + t * A.q_stride + (long long)hd * D;
    uint16_t* dst = A.q_out + t * A.q_out_stride + (long long)hd * D;
    if (A.q_vec) {  // two chunks of eight whose components are each other's partners, or neighbours where nothing is turned
      const bool turned = turn && 16 * i < A.rope_dim;
      const int c0 = turned && !A.interleaved ? 8 * i : 16 * i, c1 = turned && !A.interleaved ? c0 + r2 : c0 + 8;
      uint4 ra = ld_stream128(src + c0), rb = ld_stream128(src + c1);
      if (turned) {
        float a[8], b[8], x[8], y[8];
        unpack8<WD>(ra, a);
        unpack8<WD>(rb, b);
        float c[8], s[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float4 e = __ldg(reinterpret_cast<const float4*>(tab + 8 * i) + h), f = __ldg(reinterpret_cast<const float4*>(tab + r2 + 8 * i) + h);
          c[4 * h] = e.x; c[4 * h + 1] = e.y; c[4 * h + 2] = e.z; c[4 * h + 3] = e.w;
          s[4 * h] = f.x; s[4 * h + 1] = f.y; s[4 * h + 2] = f.z; s[4 * h + 3] = f.w;
        }
        if (A.interleaved) {
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
      continue;
    }
    for (int e = 8 * i; e < 8 * i + 8; ++e) {  // pair by pair: any alignment, any even rope_dim
      const int d0 = A.rope_dim > 0 && !A.interleaved && e < r2 ? e : 2 * e, d1 = A.rope_dim > 0 && !A.interleaved && e < r2 ? e + r2 : 2 * e + 1;
      const uint16_t a = src[d0], b = src[d1];
      if (turn && e < r2) {
        const float x1 = widen<WD>(a), x2 = widen<WD>(b), c = tab[e], s = tab[r2 + e];
        dst[d0] = narrow<WD>(x1 * c - x2 * s);
        dst[d1] = narrow<WD>(x2 * c + x1 * s);
      } else {
        dst[d0] = a;
        dst[d1] = b;
      }
    }
  }
}

// Rows of `n` elements (a multiple of 64) to where they lie side by side, at a multiple of 16 bytes.
template <int N = 256>
__global__ void __launch_bounds__(N) ls_kv4_align_kernel(const uint16_t* from, int64_t stride, uint16_t* to, int n) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  from += blockIdx.x * stride;
  to += (int64_t)blockIdx.x * n;
  for (int i = threadIdx.x; i < n; i += N) to[i] = from[i];
}

struct Kv4ReadArgs {
  Kv4Pages p;
  uint16_t* k;  // [n_tokens][kv_heads][dim], either may be NULL
  uint16_t* v;
  const int32_t* seq;
  const int32_t* pos;
  int64_t k_stride, v_stride;
  int32_t n_tokens, per_block, vec;
};

// Eight codes of a word as scale * code + zero (exact but for the last rounding of the sum), rounded to the type.
template <int WD>
__device__ __forceinline__ uint4 word_values(uint32_t w, uint32_t meta_lo, uint32_t meta_hi) {
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t m = e < 4 ? meta_lo : meta_hi;
    const float code = __uint_as_float((w >> (4 * e) & 15u) | 0x4b000000u) - 8388608.f;
    x[e] = fmaf(code, widen<WD>((uint16_t)m), widen<WD>((uint16_t)(m >> 16)));
  }
  return make_uint4(pack2<WD>(x[0], x[1]), pack2<WD>(x[2], x[3]), pack2<WD>(x[4], x[5]), pack2<WD>(x[6], x[7]));
}

__device__ __forceinline__ void put8(uint16_t* dst, uint4 v, bool vec) {
  if (vec) { *reinterpret_cast<uint4*>(dst) = v; return; }
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 8; ++e) dst[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
}

// A thread takes two words of a row at a time: 16 components of a key, or twice 8 of a value, each stored as 16 bytes.
template <int WD, int D>
__global__ void __launch_bounds__(256) ls_kv4_read_kernel(const Kv4ReadArgs A) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  constexpr int per = D / 16;
  const int items = A.p.kv_heads * 2 * per, groups = D / A.p.group, n = min(A.per_block, A.n_tokens - (int)blockIdx.x * A.per_block) * items;
  for (int x = threadIdx.x; x < n; x += 256) {
    const int tt = x / items, y = x - tt * items;
    const int j = y % per, value = y / per % 2, h = y / (2 * per);
    const long long t = (long long)blockIdx.x * A.per_block + tt;
    uint16_t* out = value ? A.v : A.k;
    if (!out) continue;
    int row = 0;
    const long long at = kv4_tile_at(A.p, A.seq[t], A.pos[t], 0x7fffffff, kv4_tile(D, A.p.group), row);
    if (at < 0) continue;
    const uint8_t* tile = A.p.pages + at + h * A.p.head_stride;
    const uint32_t* codes = reinterpret_cast<const uint32_t*>(tile + (16 * value + row) * (D / 2));
    const uint32_t* meta = reinterpret_cast<const uint32_t*>(tile + 16 * D) + (16 * value + row) * groups;
    out += t * (value ? A.v_stride : A.k_stride) + (long long)h * D;
    if (value) {
      const int g = 2 * (j % 4), ws = j / 4, lo = 64 * ws + 4 * g;
      const uint32_t a = codes[value_word<D>(g, ws, row)], b = codes[value_word<D>(g + 1, ws, row)];
      const uint32_t m0 = meta[lo / A.p.group], m1 = meta[(lo + 32) / A.p.group];
      put8(out + lo, word_values<WD>((a & 0xffffu) | b << 16, m0, m0), A.vec);
      put8(out + lo + 32, word_values<WD>(a >> 16 | (b & 0xffff0000u), m1, m1), A.vec);
    } else {
      const uint32_t a = codes[key_word<D>(2 * j, row)], b = codes[key_word<D>(2 * j + 1, row)], m = meta[16 * j / A.p.group];
      put8(out + 16 * j, word_values<WD>(a, m, m), A.vec);
      put8(out + 16 * j + 8, word_values<WD>(b, m, m), A.vec);
    }
  }
}

}  // namespace ls
