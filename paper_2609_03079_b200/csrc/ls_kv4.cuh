// A paged key/value cache held in 4 bits: where its parts lie, the append that quantises into it, the kernel that reads it back.
//
// `group` (32, 64 or 128) consecutive components of one token's key or value of one head share a scale and a zero of the cache's
// 16-bit type.  With x the components as a 16-bit cache would hold them (a key is turned in 64 bits, then rounded to 32 and to 16):
//   zero = min x;  scale = (max x - min x) / 15, each step in fp32, rounded to the type;  code = min(15, round((x - zero) / scale)), the
// difference in fp32, the exact quotient of that, ties to even
// and scale * code + zero is what is held.  scale 0: all codes are 0.  A range that is not finite: scale and zero are NaN.
// Every step is rounded as said and no other, so that codes do not depend on who computes them.
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

// Eight consecutive components.
__device__ __forceinline__ uint4 load_oct(const uint16_t* p, bool vec) {
  if (vec) return ld_stream128(p);
  return make_uint4(p[0] | (uint32_t)p[1] << 16, p[2] | (uint32_t)p[3] << 16, p[4] | (uint32_t)p[5] << 16, p[6] | (uint32_t)p[7] << 16);
}
// The larger of each half; NaN if either is.
template <int WD>
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  uint32_t r;
  if (WD == WD_BF16) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Where a lane's eight components (8 oct ...) of a row go in a tile: the word that it stores, and its group's scale and zero.
template <int D, int G>
struct OctPlace {
  int word, meta;
  bool leads, high;  // its group's scale is this lane's to store; (values) its components are the high halves of their words
  __device__ __forceinline__ OctPlace(bool value, int oct, int row) {
    leads = oct % (G / 8) == 0;
    high = oct & 4;
    word = ((value ? 16 : 0) + row) * (D / 2) + 4 * (value ? value_word<D>(oct % 4 * 2 + high, oct >> 3, row) : key_word<D>(oct, row));
    meta = 16 * D + (((value ? 16 : 0) + row) * (D / G) + oct / (G / 8)) * 4;
  }
};

// Quantises the lane's eight components (as the type holds them) with the other lanes of their group, and stores them in `tile` (NULL:
// nowhere).
template <int WD, int D, int G>
__device__ __forceinline__ void store_oct(uint4 x, bool value, const OctPlace<D, G>& at, uint8_t* tile) {
  // (-min, max) of the group, both as maxima of 16-bit halves
  const uint32_t neg = 0x80008000u;
  uint32_t m;
  {
    const uint32_t up = max2<WD>(max2<WD>(x.x, x.y), max2<WD>(x.z, x.w)), down = max2<WD>(max2<WD>(x.x ^ neg, x.y ^ neg), max2<WD>(x.z ^ neg, x.w ^ neg));
    m = max2<WD>(__byte_perm(down, up, 0x5410), __byte_perm(down, up, 0x7632));
#pragma unroll
    for (int o = 1; o < G / 8; o <<= 1) m = max2<WD>(m, __shfl_xor_sync(0xffffffffu, m, o));
  }
  const float lo = -widen<WD>((uint16_t)m), range = widen<WD>((uint16_t)(m >> 16)) - lo;
  const bool fine = range < INFINITY;
  // range / 15, correctly rounded: the product with 1 / 15 put right by its remainder (P. W. Markstein, IBM J. Res. Dev. 34, 1990), the same as the
  // quotient for all 2^23 fractions
  const float fifteenth = 0.0666666701436042785645f, about = __fmul_rn(range, fifteenth);
  const uint16_t scale16 = narrow<WD>(__fmaf_rn(__fmaf_rn(-15.f, about, range), fifteenth, about));
  const float scale = fine ? widen<WD>(scale16) : 0.f;
  // (x - zero) / scale to the nearest whole number, ties to even: by a reciprocal, then put right by the remainder, which is exact (a
  // whole number up to 16 times a 16-bit scale fits fp32, and what is left of x - zero is at most about half a scale).
  // A division's quotient, where reciprocals end, needs none: a number that is not halfway between two codes times the scale is a last place off it at
  // least, and so is its quotient.  (Deciding ties by what x - zero lost when it was rounded, where exponents are far apart: 128 us for 16
  // chunks of 1023 tokens, 117 without.)
  float y[8];
  unpack8<WD>(x, y);
  const float inverse = __fdividef(1.f, scale), magic = 12582912.f;
  float c[8], over = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    y[e] = __fsub_rn(y[e], lo);
    c[e] = __fmaf_rn(y[e], inverse, magic);  // (whole, in the low bits)
    over = fmaxf(over, fabsf(fmaf(-__fsub_rn(c[e], magic), scale, y[e])));
  }
  if (!(scale > 1e-30f)) {  // (reciprocals end there; a scale of 0 or NaN: codes of 0)
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = magic + (scale > 0.f ? rintf(__fdiv_rn(y[e], scale)) : 0.f);
  } else if (2.f * over >= scale) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float r = fmaf(-__fsub_rn(c[e], magic), scale, y[e]), past = fmaf(2.f, fabsf(r), -scale);
      if (past > 0.f || (past == 0.f && (__float_as_uint(c[e]) & 1))) c[e] += r > 0.f ? 1.f : -1.f;
    }
  }
  uint32_t codes = 0;
#pragma unroll
  for (int e = 7; e >= 0; --e) codes = codes * 16 + __float_as_uint(fminf(c[e], magic + 15.f));
  codes -= 0x4b400000u * 0x11111111u;
  if (value) {  // components 32 apart share a word: the lower four of each are one lane's word, the upper four the other's
    const uint32_t other = __shfl_xor_sync(0xffffffffu, codes, 4);
    codes = at.high ? __byte_perm(other, codes, 0x7632) : __byte_perm(codes, other, 0x5410);
  }
  if (!tile) return;
  *reinterpret_cast<uint32_t*>(tile + at.word) = codes;
  if (at.leads) *reinterpret_cast<uint32_t*>(tile + at.meta) = fine ? scale16 | ((m ^ 0x8000u) & 0xffffu) << 16 : 0x7fff7fffu;
}

// Cosines and signed sines of the lane's components, and their partners.
struct Turn { float c[8], s[8]; };
__device__ __forceinline__ Turn turn_of(const Kv4AppendArgs& A, int d0, const float* tab) {
  const int r2 = A.rope_dim / 2;
  Turn t;
  if (A.rope_vec) {  // half of the turned part is a multiple of eight: partners and angles are eights too
    const bool far = !A.interleaved && d0 >= r2;
    const float4* at = reinterpret_cast<const float4*>(tab + (A.interleaved ? d0 / 2 : far ? d0 - r2 : d0));
    const float4 c = __ldg(at), s = __ldg(at + r2 / 4);
    if (A.interleaved) {
      const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) { t.c[e] = cc[e / 2]; t.s[e] = e & 1 ? ss[e / 2] : -ss[e / 2]; }
    } else {
      const float4 c1 = __ldg(at + 1), s1 = __ldg(at + 1 + r2 / 4);
      const float cc[8] = {c.x, c.y, c.z, c.w, c1.x, c1.y, c1.z, c1.w}, ss[8] = {s.x, s.y, s.z, s.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) { t.c[e] = cc[e]; t.s[e] = far ? ss[e] : -ss[e]; }
    }
    return t;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int d = d0 + e, j = A.interleaved ? d / 2 : d < r2 ? d : d - r2;
    t.c[e] = 1.f; t.s[e] = 0.f;
    if (d >= A.rope_dim) continue;
    t.c[e] = tab[j];
    t.s[e] = (A.interleaved ? d & 1 : d >= r2) ? tab[r2 + j] : -tab[r2 + j];
  }
  return t;
}
__device__ __forceinline__ uint4 load_partners(const Kv4AppendArgs& A, const uint16_t* head, int d0, uint4 mine) {
  const int r2 = A.rope_dim / 2;
  if (A.interleaved)
    return make_uint4(__byte_perm(mine.x, 0, 0x1032), __byte_perm(mine.y, 0, 0x1032), __byte_perm(mine.z, 0, 0x1032), __byte_perm(mine.w, 0, 0x1032));
  if (A.rope_vec) return load_oct(head + (d0 < r2 ? d0 + r2 : d0 - r2), A.kv_vec);
  uint32_t x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int d = d0 + e;
    x[e] = d >= A.rope_dim ? 0 : head[d < r2 ? d + r2 : d - r2];
  }
  return make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16);
}
// x c + partner s, as the 16-bit type holds it.  The sum of the two products is taken exactly but for 2^-48 of it (each product as two
// fp32 numbers, their sum with its error) and rounded to fp32 once, then to the type: keys, and with them codes, are those of 64-bit
// arithmetic, without its conversions, which kept the conversion units busy.
template <int WD>
__device__ __forceinline__ uint4 turned_oct(uint4 mine, uint4 partners, const Turn& t) {
  float a[8], b[8];
  unpack8<WD>(mine, a);
  unpack8<WD>(partners, b);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float p = __fmul_rn(a[e], t.c[e]), q = __fmul_rn(b[e], t.s[e]);
    const float low = __fadd_rn(__fmaf_rn(a[e], t.c[e], -p), __fmaf_rn(b[e], t.s[e], -q));
    const float sum = __fadd_rn(p, q), back = __fsub_rn(sum, p);
    const float lost = __fadd_rn(__fsub_rn(p, __fsub_rn(sum, back)), __fsub_rn(q, back));
    const float z = __fadd_rn(sum, __fadd_rn(lost, low));
    a[e] = fabsf(sum) < INFINITY ? z : sum;
  }
  return make_uint4(pack2<WD>(a[0], a[1]), pack2<WD>(a[2], a[3]), pack2<WD>(a[4], a[5]), pack2<WD>(a[6], a[7]));
}

// Slabs of 256 components that a warp takes of a token's keys or values, eight to a lane, and heads of queries that each lane takes 16
// components of.  More of them share a lane's angles and keep more loads on their way; fewer leave more warps.  In us, 16 chunks of 1023 tokens, 64 / 8
// heads of 128 (floor 98): slabs 1, 2, 4: 130, 117, 134; heads 1, 2, 4: 162, 129, 117.  One token: 2.6, 3.0, 4.6; 2.9, 3.0, 3.0.
constexpr int K4_SLABS = 2;
constexpr int K4_Q_HEADS = 4;

// A warp takes K4_SLABS slabs of a token's keys or of its values, or 512 K4_Q_HEADS components of its queries; a lane's angles are the
// same in all of them.  Queries are turned in fp32 and rounded once, as in the 16-bit append.
// Bound by memory: 117 us for the chunks above, 0.84 of the rate of a copy; with as many key heads as query heads (4 chunks of 1023, 40 / 40 heads)
// by the arithmetic of the keys' codes, 80 us for a floor of 30.  Four CTAs to an SM (3: 129 us, 5: 192, which spills).  Operands that do not lie
// at multiples of 16 bytes are read element by element: 439 us.
template <int WD, int D, int G>
__global__ void __launch_bounds__(256, 4) ls_kv4_append_kernel(const Kv4AppendArgs A) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int lane = threadIdx.x & 31;
  const uint32_t id = blockIdx.x * 8 + (threadIdx.x >> 5);
  const long long t = id / (uint32_t)A.jobs;
  const int job = (int)(id - (uint32_t)t * (uint32_t)A.jobs);
  if (t >= A.n_tokens) return;
  if (job < 2 * A.kv_jobs) {
    const bool value = job >= A.kv_jobs;
    const int oct = lane % (D / 8), step = 256 / D, h0 = K4_SLABS * (value ? job - A.kv_jobs : job) * step + lane / (D / 8);
    const uint16_t* token = (value ? A.v + t * A.v_stride : A.k + t * A.k_stride) + 8 * oct;
    const bool turn = !value && 8 * oct < A.rope_dim;
    uint4 mine[K4_SLABS], other[K4_SLABS];
    auto source = [&](int i) { return token + (long long)min(h0 + i * step, A.p.kv_heads - 1) * D; };
#pragma unroll
    for (int i = 0; i < K4_SLABS; ++i) mine[i] = load_oct(source(i), A.kv_vec);
    const int sq = A.seq[t], ps = A.pos[t];
    if (turn) {
#pragma unroll
      for (int i = 0; i < K4_SLABS; ++i) other[i] = load_partners(A, source(i) - 8 * oct, 8 * oct, mine[i]);
    }
    int row = 0;
    const long long at = kv4_tile_at(A.p, sq, ps, A.rope_dim > 0 ? A.rope_positions : 0x7fffffff, kv4_tile(D, G), row);
    if (at < 0) return;
    if (turn) {
      const Turn angle = turn_of(A, 8 * oct, A.rope + (long long)ps * A.rope_dim);
#pragma unroll
      for (int i = 0; i < K4_SLABS; ++i) {
        const uint4 b = turned_oct<WD>(mine[i], other[i], angle);
        const int left = A.rope_vec ? 8 : A.rope_dim - 8 * oct;  // (whole pairs are turned; the rest stays as it is)
        mine[i].x = b.x;
        if (left > 2) mine[i].y = b.y;
        if (left > 4) mine[i].z = b.z;
        if (left > 6) mine[i].w = b.w;
      }
    }
    const OctPlace<D, G> place(value, oct, row);
    uint8_t* tile = A.p.pages + at;
#pragma unroll
    for (int i = 0; i < K4_SLABS; ++i) {
      const int h = h0 + i * step;
      if (h - lane / (D / 8) >= A.p.kv_heads) break;
      store_oct<WD, D, G>(mine[i], value, place, h < A.p.kv_heads ? tile + h * A.p.head_stride : nullptr);
    }
    return;
  }
  const int ps = A.pos[t], r2 = A.rope_dim / 2;
  const bool turn = A.rope_dim > 0 && ps >= 0 && ps < A.rope_positions;
  const float* tab = A.rope + (long long)ps * A.rope_dim;
  const int i = lane % (D / 16), h0 = (job - 2 * A.kv_jobs) * (K4_Q_HEADS * 512 / D) + lane / (D / 16), step = 512 / D;
  const uint16_t* src = A.q + t * A.q_stride;
  uint16_t* dst = A.q_out + t * A.q_out_stride;
  if (A.q_vec) {  // two chunks of eight whose components are each other's partners, or neighbours where nothing is turned
    const bool turned = turn && 16 * i < A.rope_dim;
    const int c0 = turned && !A.interleaved ? 8 * i : 16 * i, c1 = turned && !A.interleaved ? c0 + r2 : c0 + 8;
    uint4 ra[K4_Q_HEADS], rb[K4_Q_HEADS];
#pragma unroll
    for (int k = 0; k < K4_Q_HEADS; ++k) {
      const uint16_t* p = src + (long long)min(h0 + k * step, A.heads - 1) * D;
      ra[k] = ld_stream128(p + c0);
      rb[k] = ld_stream128(p + c1);
    }
    float c[8], s[8];
    if (turned) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float4 e = __ldg(reinterpret_cast<const float4*>(tab + 8 * i) + h), f = __ldg(reinterpret_cast<const float4*>(tab + r2 + 8 * i) + h);
        c[4 * h] = e.x; c[4 * h + 1] = e.y; c[4 * h + 2] = e.z; c[4 * h + 3] = e.w;
        s[4 * h] = f.x; s[4 * h + 1] = f.y; s[4 * h + 2] = f.z; s[4 * h + 3] = f.w;
      }
    }
#pragma unroll
    for (int k = 0; k < K4_Q_HEADS; ++k) {
      if (h0 + k * step >= A.heads) break;
      uint16_t* out = dst + (long long)(h0 + k * step) * D;
      if (turned) {
        float a[8], b[8], x[8], y[8];
        unpack8<WD>(ra[k], a);
        unpack8<WD>(rb[k], b);
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
        ra[k] = make_uint4(pack2<WD>(x[0], x[1]), pack2<WD>(x[2], x[3]), pack2<WD>(x[4], x[5]), pack2<WD>(x[6], x[7]));
        rb[k] = make_uint4(pack2<WD>(y[0], y[1]), pack2<WD>(y[2], y[3]), pack2<WD>(y[4], y[5]), pack2<WD>(y[6], y[7]));
      }
      *reinterpret_cast<uint4*>(out + c0) = ra[k];
      *reinterpret_cast<uint4*>(out + c1) = rb[k];
    }
    return;
  }
  for (int k = 0; k < K4_Q_HEADS; ++k) {
    const int hd = h0 + k * step;
    if (hd >= A.heads) return;
    const uint16_t* from = src + (long long)hd * D;
    uint16_t* out = dst + (long long)hd * D;
    for (int e = 8 * i; e < 8 * i + 8; ++e) {  // pair by pair: any alignment, any even rope_dim
      const int d0 = A.rope_dim > 0 && !A.interleaved && e < r2 ? e : 2 * e, d1 = A.rope_dim > 0 && !A.interleaved && e < r2 ? e + r2 : 2 * e + 1;
      const uint16_t a = from[d0], b = from[d1];
      if (turn && e < r2) {
        const float x1 = widen<WD>(a), x2 = widen<WD>(b), c = tab[e], s = tab[r2 + e];
        out[d0] = narrow<WD>(x1 * c - x2 * s);
        out[d1] = narrow<WD>(x2 * c + x1 * s);
      } else {
        out[d0] = a;
        out[d1] = b;
      }
    }
  }
}

// Rows of `n` elements (a multiple of 64) to where they lie side by side, at a multiple of 16 bytes: queries that the attention could
// not load 16 bytes at a time.
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
  int32_t n_tokens, width, vec;  // width: threads of a token
};

// Pairs of codes as scale * code + zero, rounded once (a fused multiply-add of the type).  The codes come as integers above 1024 (fp16)
// or 128 (bf16), from which the type's own subtraction takes them exactly.
template <int WD>
__device__ __forceinline__ uint32_t pair_values(uint32_t codes, uint32_t scale, uint32_t zero) {
  uint32_t u, r;
  if (WD == WD_BF16) {
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(u) : "r"(codes | 0x43004300u), "r"(0x43004300u));
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(u), "r"(scale), "r"(zero));
  } else {
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(u) : "r"(codes | 0x64006400u), "r"(0x64006400u));
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(u), "r"(scale), "r"(zero));
  }
  return r;
}
// The eight codes of a word, in order.
template <int WD>
__device__ __forceinline__ uint4 word_values(uint32_t w, uint32_t meta) {
  const uint32_t scale = __byte_perm(meta, 0, 0x1010), zero = __byte_perm(meta, 0, 0x3232);
  uint32_t r[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = pair_values<WD>(w >> (4 * e) & 0x000f000fu, scale, zero);
  return make_uint4(__byte_perm(r[0], r[1], 0x5410), __byte_perm(r[2], r[3], 0x5410), __byte_perm(r[0], r[1], 0x7632), __byte_perm(r[2], r[3], 0x7632));
}

__device__ __forceinline__ void put8(uint16_t* dst, uint4 v, bool vec) {
  if (vec) { *reinterpret_cast<uint4*>(dst) = v; return; }
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 8; ++e) dst[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
}

// `width` threads to a token, each with 16 components of a key and of a value of every head that it visits: two words of each, stored
// as two times 16 bytes.  Bound by memory, four fifths of it writes: 134 us for 16 sequences of fp16 with a floor of 109; rows that do not
// lie at multiples of 16 bytes are written element by element (1261 us).
template <int WD, int D>
__global__ void __launch_bounds__(256) ls_kv4_read_kernel(const Kv4ReadArgs A) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  constexpr int per = D / 16;
  const int tt = threadIdx.x / A.width, y0 = threadIdx.x - tt * A.width, items = A.p.kv_heads * per, groups = D / A.p.group;
  const long long t = (long long)blockIdx.x * (256 / A.width) + tt;
  if (tt >= 256 / A.width || t >= A.n_tokens) return;
  int row = 0;
  const long long at = kv4_tile_at(A.p, A.seq[t], A.pos[t], 0x7fffffff, kv4_tile(D, A.p.group), row);
  if (at < 0) return;
  const uint32_t* codes = reinterpret_cast<const uint32_t*>(A.p.pages + at) + row * (D / 8);
  const uint32_t* meta = reinterpret_cast<const uint32_t*>(A.p.pages + at + 16 * D) + row * groups;
  uint16_t *k_out = A.k + t * A.k_stride, *v_out = A.v + t * A.v_stride;
  const int shift = A.p.group == 32 ? 5 : A.p.group == 64 ? 6 : 7;
#pragma unroll 2
  for (int y = y0; y < items; y += A.width) {
    const int h = y / per, j = y % per, g = 2 * (j % 4), ws = j / 4, lo = 64 * ws + 4 * g;
    const long long to = h * A.p.head_stride / 4;
    if (A.k) {
      const uint32_t a = __ldg(codes + to + key_word<D>(2 * j, row)), b = __ldg(codes + to + key_word<D>(2 * j + 1, row)), m = __ldg(meta + to + (16 * j >> shift));
      put8(k_out + h * D + 16 * j, word_values<WD>(a, m), A.vec);
      put8(k_out + h * D + 16 * j + 8, word_values<WD>(b, m), A.vec);
    }
    if (A.v) {
      const uint32_t a = __ldg(codes + to + 2 * D + value_word<D>(g, ws, row)), b = __ldg(codes + to + 2 * D + value_word<D>(g + 1, ws, row));
      const uint32_t m0 = __ldg(meta + to + 16 * groups + (lo >> shift)), m1 = __ldg(meta + to + 16 * groups + ((lo + 32) >> shift));
      put8(v_out + h * D + lo, word_values<WD>(__byte_perm(a, b, 0x5410), m0), A.vec);
      put8(v_out + h * D + lo + 32, word_values<WD>(__byte_perm(a, b, 0x7632), m1), A.vec);
    }
  }
}

}  // namespace ls
