// Attention over the 4-bit paged cache: queries of a few tokens per sequence against all of its keys.
//
// With u the codes and (s, z) scale and zero of a group, key j and value j are s_j u_j + z_j, so that (sums over groups left out)
//   score_j = scale (s_j <q, u_j> + z_j sum(q)),   out = (sum_j p_j s_j u_j + sum_j p_j z_j) / sum_j p_j,   p_j = e^(score_j - M).
// Both products take the codes themselves: four bits in the mantissa of a 16-bit float with an exponent of zero are a subnormal
// number, u 2^-24 times their place, exact in the tensor cores, so a word of eight codes becomes four operand registers with a few
// shifts and logical instructions and no conversion.  The sums of a product are aligned to 2^-14, not to what the subnormal numbers come
// to, so a code at bit 0 loses what lies below 2^-14 of a unit (lse was off by 4e-6): they stand at bits 2 and 6 (2^-16; the 2^-4 between the
// two goes into the query, and into the sums of values when they are done).
// Queries are scaled to a power of two per row and are exact in fp16, whatever the cache's type (but for bf16 components about 2^27 and more below
// the row's largest, which lose bits).  A row's tensor-core work is a small part
// of its instructions: 16 keys cost about 251 instructions of a warp (a scale for 128 components, up to 8 rows), 296 (for 64) or 437 (for 64, 16 rows).
//
// Bounds and figures (B200, passes among others):
//   128 sequences of up to 9216 keys, 64 / 8 heads of 128, one scale a head: 169 to 180 us where seconds of such calls meet the card's power
//     limit, 0.70 to 0.74 of the rate at which memory is copied, and 158 in bursts, 0.79; 16 of 400001 keys 765 us, 0.89;
//   one sequence of 100001 keys 33 us; two million keys 438, 0.81 (0.84 from one to the other): about 12 us of a call are its beginning
//     (lengths, shares, table, first tile, all of it cold code) and its end (the team's sums, then the joining of a unit's pieces);
//   33 sequences of up to 2000 keys, 40 / 40 heads, a scale for 32: 60 us, 0.70, 64 at the power limit (80 us with a column for a row, of which seven
//     in eight are idle, and a sum for each group);
//   16 rows (draft tokens): 16 sequences of a window of 4096 35 us, 0.26, two warps to a scheduler.
// What did not help (all measured on earlier forms): a software pipeline of scores and values (170 us for 174, others slower), codes brought to
// their bits by byte permutations (the same within 1 %) or by the high half of a product (5 to 15 % slower) instead of right shifts, scores of 32 rows at
// once (163 us for two passes' 100).
#pragma once
#include "ls_attend.cuh"
#include "ls_kv4.cuh"
#include "ls_tmem.cuh"

namespace ls {

// n / d for 0 <= n < 2^31 by a multiplication: mul = ceil(2^shift / d), shift = 31 + ceil(log2 d).
struct FastDiv {
  uint32_t mul, shift;
  __device__ __forceinline__ int operator()(int n) const { return (int)((uint64_t)(uint32_t)n * mul >> shift); }
};

struct Attend4Args {
  Kv4Pages p;
  const uint16_t* q;   // [n_seqs * q_len][heads][dim], token stride q_stride
  uint16_t* out;
  float* lse;          // [n_seqs * q_len][heads] or NULL
  const int32_t* seq_len;
  float* part;         // pieces of rows: [2 * teams][rows of a unit][dim + 4]: sums of values, then M (log 2) and the sum of weights
  int32_t* arrived;    // [units], zero between calls: pieces that are written
  int64_t q_stride, out_stride;
  int32_t q_len, heads, group, window, row_tiles, out_vec;
  int32_t most, behind;  // positions that a sequence can have; of those, how many from its end on are seen by any of its tokens
  FastDiv by_group, by_row_tiles, by_page;  // (by_page: tiles of a page)
  float scale_log2;
};

constexpr long long K4_SPIN_CLOCKS = 4000000000LL;  // about two seconds
// What a unit's beginning and end, and the joining of its pieces, cost a warp, in tiles.  (A unit at 4, 6, 8 and 11: one sequence of 100001 keys 35.9, 33.4,
// 33.1, 32.9 us; 33 of up to 2000 59.1, 59.4, 59.8, 61.3; three of 20001 21.1, 20.1, 18.9, 18.7; 200 of 300 22.1, 22.2, 22.2, 22.1; a window of 4096, 16 rows, 36.0, 36.3,
// 34.6, 35.1; 128 long ones 156, 155, 158, 158; 200 tiny ones and a long one 36, 41, 40, 41.)
constexpr float K4_UNIT_TILES = 8.f, K4_JOIN_TILES = 4.f, K4_ADD_TILES = 3e-4f;
// Blocks that one call may deal out (they are counted in 32 bits); the host cuts larger batches.
constexpr long long K4_MAX_BLOCKS = 1LL << 30;
constexpr float K4_FACTOR = 0x1p60f, K4_LEAST_FACTOR = 0x1p-100f;  // bounds of the factors of scales (their reciprocals, times 2^22, fit fp32)
// The products' sums are truncated each time: what they hold is brought to the middle of the codes every K4_MIDDLE blocks, and a warp's sums end after
// K4_RUN blocks, to be added up by rounded operations.  (Without either a warp that summed 2^19 keys was off by 4 % of a mean of values.  Every 8, 32, 64
// blocks, in us: 128 long 159.6, 158.2, 159.0; 33 conversations 60.1, 59.9, 59.8, and 58.1 without.  Runs of 512 blocks or none: 16 sequences of 400001 keys 765
// and 762 us.  Runs of 64 or 128 instead of both: 801, 787; 128 long 164.8, 159.5; 33 conversations 59.2, 59.2.)
constexpr int K4_MIDDLE = 32, K4_RUN = 512;

// Shapes of the kernel: D components a head, groups of G, NT times 8 rows of queries at once.  Up to 8 rows are the columns of the
// products (S^T = K Q^T, O^T = V^T P^T: the codes are the operand with 16 rows), 16 rows are their rows (S = Q K^T, O = P V).
// NT = 0: so few rows that the 8 columns hold each of them once for every group, with the components of that group alone.  One sum then
// holds what a scale and a zero have to be applied to, two columns to a lane, instead of one sum for each group.  (In us, with and
// without: 33 sequences of up to 2000 keys, one row, four groups: 59.8, 80.3; 8 of 8001, one row, two groups: 45.1, 47.8; 200 of 300 keys, four
// rows, two groups: 22.2, 23.9; 200 of 17 and one of 40000: 40.3, 38.7.)
template <int D, int G, int NT>
struct K4Shape {
  // 12 warps of 168 registers, or 8 of 255 where sums fill more.  Two tiles at once give a warp independent work (in us, warps x tiles; up to
  // 8 rows of heads of 128: 12 x 2, 8 x 2, 16 x 2, 16 x 1: 128 long sequences 158, 184, 156, 200; one of 100001 33, 35, 39, 38; 33 of up to 2000 60, 66, 57, 67;
  // 200 of 300 keys 22, 28, 24, 26; 16 of 20001, a scale for 32: 71, 70, 95, 91.  16 rows, window of 4096: 8 x 2, 8 x 1, 12 x 1, 10 x 2: 35, 37, 51, 60).
  static constexpr int N8 = NT == 2 ? 2 : 1;
  static constexpr int WARPS = D * N8 <= 128 ? 12 : 8;
  static constexpr int KT = D == 256 && G == 32 ? 1 : 2;         // (two would spill 660 bytes a thread, one 180)
  static constexpr int THREADS = WARPS * 32;
  static constexpr int NG = D / G;
  static constexpr int ROWS = NT == 0 ? 8 / NG : 8 * NT;
  static constexpr int TILE = kv4_tile(D, G);
  static constexpr int LINE = D + 4;                     // floats of a row's piece
  static constexpr int PIECE = ROWS * LINE * 4;
  // Operands of the queries stay in registers, or, where sums of values fill those, in shared memory (each lane's own).
  static constexpr bool Q_SHARED = NT > 1;
  static constexpr int Q_BYTES = Q_SHARED ? NT * (D / 32) * 512 : 0;
  static constexpr int FIT = (232448 - 256 - WARPS * (64 + Q_BYTES)) / (WARPS * KT * TILE);
  static constexpr int STAGES = FIT < 8 ? FIT : 8;
  // a warp's ring of blocks; once it is empty, at a unit's end, the same place holds the warp's piece
  // (three of the smallest team at least, where a unit's are fetched)
  static constexpr int LEAST = Q_SHARED ? 2 : 1;
  static constexpr int ENOUGH = (3 * PIECE / LEAST + 127) / 128 * 128;
  static constexpr int RING = STAGES * KT * TILE > ENOUGH ? STAGES * KT * TILE : ENOUGH;
  static constexpr int SMEM = WARPS * (RING + Q_BYTES + 64) + 256;
  static_assert(STAGES >= 2 && SMEM <= 232448, "ring");
};

// D = A B + (first ? 0 : D).
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, bool first = false) {
  if (first)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t halves(float lo, float hi) { return pack2<WD_FP16>(lo, hi); }
template <int WD>
__device__ __forceinline__ float2 both_halves(uint32_t m) {
  if (WD == WD_BF16) return make_float2(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&m));
}
template <int N>
__device__ __forceinline__ void lds_words(const uint8_t* p, uint32_t (&w)[N]) {
  if constexpr (N == 1) w[0] = *reinterpret_cast<const uint32_t*>(p);
  else if constexpr (N == 2) { const uint2 v = *reinterpret_cast<const uint2*>(p); w[0] = v.x; w[1] = v.y; }
  else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const uint4 v = *reinterpret_cast<const uint4*>(p + 16 * i);
      w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
    }
  }
}
__device__ __forceinline__ float quad_sum(float x) {  // over the four lanes of a row
  x += __shfl_xor_sync(0xffffffffu, x, 1);
  return x + __shfl_xor_sync(0xffffffffu, x, 2);
}
__device__ __forceinline__ float quad_max(float x) {
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
  return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
}
__device__ __forceinline__ float rows_sum(float x) {  // over the eight lanes of a column
  x += __shfl_xor_sync(0xffffffffu, x, 4);
  x += __shfl_xor_sync(0xffffffffu, x, 8);
  return x + __shfl_xor_sync(0xffffffffu, x, 16);
}
__device__ __forceinline__ float rows_max(float x) {
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
  return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
}
// (m, l, v) += a piece: its reference, its sum of weights, four of its sums.
__device__ __forceinline__ void k4_add(float& m, float& l, float4& v, float m1, float l1, float4 v1) {
  const float to = fmaxf(m, m1), f = ex2(m - to), g = ex2(m1 - to);
  m = to;
  l = fmaf(g, l1, l * f);
  v = make_float4(fmaf(g, v1.x, v.x * f), fmaf(g, v1.y, v.y * f), fmaf(g, v1.z, v.z * f), fmaf(g, v1.w, v.w * f));
}

// What has to be read of a sequence of n positions: its first block (16 KT keys) and its number of blocks.
__device__ __forceinline__ int k4_len(const Attend4Args& A, int n) { return min(max(n, 0), A.most); }
template <int KT>
__device__ __forceinline__ int k4_first(const Attend4Args& A, int n) { return max(0, n - A.behind) / (16 * KT); }
template <int KT>
__device__ __forceinline__ int k4_blocks(const Attend4Args& A, int n) { return (n + 16 * KT - 1) / (16 * KT) - k4_first<KT>(A, n); }

// A unit is one sequence's blocks (16 KT keys each) for one key head and one row tile of its queries.  All units' blocks stand in one line,
// cut into equal shares; a share belongs to a team (a whole CTA, or 4, 2 or 1 of its warps), which deal out its blocks among themselves.  A warp copies its
// blocks by itself (bulk copies into a ring of its own) and works alone until a unit's end (or that of a run of K4_RUN blocks); then the team adds up, and a unit that
// reaches over several teams is joined, in order, by whichever of them comes last.
// A call's first pass over any code waits for it to come from L2, which is most of a small call: loops that need not be unrolled are not.
template <int WD, int D, int G, int NT>
__global__ void __launch_bounds__(K4Shape<D, G, NT>::THREADS, 1) ls_kv4_attend_kernel(const __grid_constant__ Attend4Args A) {
  using S = K4Shape<D, G, NT>;
  constexpr int NG = S::NG, NW = D / 64, KW = D / 32, ST = S::STAGES, KT = S::KT;
  constexpr int N8 = S::N8;
  constexpr bool WIDE = NT == 2, COLS = NT == 0;
  constexpr int NS = COLS ? 1 : NG, NV = COLS ? 2 : NG, NR = COLS ? 1 : 2;  // sums of scores, scales of a token that are the lane's, rows of the lane
  extern __shared__ __align__(128) uint8_t smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  uint8_t* ring = smem + warp * S::RING;
  uint8_t* q_shared = smem + S::WARPS * S::RING + warp * S::Q_BYTES + lane * 16;
  uint8_t* rest = smem + S::WARPS * (S::RING + S::Q_BYTES);
  const uint32_t bar = saddr(rest + warp * 64);
  int* s_last = reinterpret_cast<int*>(rest + S::WARPS * 64);  // [WARPS]
  int* s_dead = s_last + S::WARPS;                             // bits by warp
  if (lane < ST) mb_init(bar + 8 * lane, 1);
  if (threadIdx.x == 0) *s_dead = 0;
  fence_async_shared();
  __syncthreads();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // All blocks of a head, and the most that a sequence has.  Every warp adds up for itself, four sequences to a lane at a time.
  const int per_seq = A.p.kv_heads * A.row_tiles, n_seqs = A.p.n_seqs;
  int total = 0, longest = 1, busy = 0;
  bool bad = false;
#pragma unroll 1
  for (int b0 = lane; b0 < n_seqs; b0 += 128) {
    int n[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) n[i] = b0 + 32 * i < n_seqs ? A.seq_len[b0 + 32 * i] : -1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int len = k4_len(A, n[i]), blocks = b0 + 32 * i < n_seqs ? k4_blocks<KT>(A, len) : 0;
      bad |= b0 + 32 * i < n_seqs && len != n[i];
      busy += blocks > 0;
      total += blocks;
      longest = max(longest, blocks);
    }
  }
  if (bad && blockIdx.x == 0 && warp == 0) set_status(A.p.status, ST_BAD_INDEX);
  total = __reduce_add_sync(0xffffffffu, total) * per_seq;
  longest = __reduce_max_sync(0xffffffffu, longest);
  busy = __reduce_add_sync(0xffffffffu, busy);
  // sequences without a key
  if (busy < n_seqs) {
#pragma unroll 1
    for (int b = blockIdx.x; b < n_seqs; b += gridDim.x) {
      if (k4_len(A, A.seq_len[b])) continue;
#pragma unroll 1
      for (long long tk = (long long)b * A.q_len; tk < (long long)(b + 1) * A.q_len; ++tk) {
#pragma unroll 1
        for (int x = threadIdx.x; x < A.heads * (D / 4); x += S::THREADS) {
          uint16_t* dst = A.out + tk * A.out_stride + 4 * x;
          if (A.out_vec) *reinterpret_cast<uint2*>(dst) = make_uint2(0, 0);
          else dst[0] = dst[1] = dst[2] = dst[3] = 0;
        }
#pragma unroll 1
        for (int x = threadIdx.x; A.lse && x < A.heads; x += S::THREADS) A.lse[tk * A.heads + x] = -INFINITY;
      }
    }
  }

  // Shares: whatever ends first, by blocks that a warp has one after another.  Either units follow each other without a gap, so that every
  // team has as much but begins and ends inside a unit; what a unit's beginning and end cost a team (K4_UNIT blocks of each warp) stands
  // in the line in front of it.  Or each unit begins with a new share, one for all of it, or several.  (Shares may be a little larger than
  // they need to be: fp32 will do.)
  // What each way is for, in us (the rule; always the first; never one share to a unit; always whole CTAs; always the smallest teams): one short
  // sequence 7.0, 9.0, 9.1, 7.0, 15; one of 100001 keys 33, 33, 33, 33, 376; 33 of up to 2000 60, 60, 60, 99, 60; a window of 4096 35, 34, 35, 35, 41; 128 long ones 158,
  // 158, 161, 177, 158; 200 of 300 22, 26, 26, 60, 22; three of 20001 19, 19, 19, 19, 75.  And without the units' own cost in the line, units' beginnings
  // pile up on some teams: 33 of up to 2000 145 us, 200 tiny ones and a long one 338 instead of 40.
  int w, share, extra;
  bool gaps;
  {  // (a lane for each size of a team)
    w = lane == 0 ? S::WARPS : max(S::LEAST, 8 >> lane);
    constexpr float K4_UNIT = K4_UNIT_TILES / KT, K4_JOIN = K4_JOIN_TILES / KT, K4_ADD = K4_ADD_TILES / KT;
    const float units = (float)(busy * per_seq), all = (float)total, above = 1.f + 1e-6f;
    const float each = __fdividef(1.f, (float)w), teams = (float)(S::WARPS / w * gridDim.x);
    const float ahead = ceilf(K4_UNIT * (float)w), even = floorf(__fdividef(all + units * ahead, teams) * above) + 1.f, some = floorf(__fdividef(all, teams - units) * above) + 1.f;
    auto join = [&](float of) {  // for every time that the team's place is filled, and for every piece that its threads add up
      const float n = __fdividef((float)longest, of) + 1.f;
      return K4_JOIN + n * each * ((float)S::PIECE / S::RING + K4_ADD * (float)(S::ROWS * D));
    };
    const float cost_even = even * each + K4_UNIT + join(even);
    const float cost_some = units < teams ? some * each + K4_UNIT + join(some) : 1e30f, cost_one = units <= teams ? longest * each + K4_UNIT : 1e30f;
    const float cost = fminf(cost_even, fminf(cost_some, cost_one));
    gaps = cost != cost_even;
    share = cost == cost_even ? (int)even : cost == cost_one ? longest : (int)some;
    const int best = __reduce_min_sync(0xffffffffu, (__float_as_uint(cost) & ~31u) | lane) & 31;
    w = __shfl_sync(0xffffffffu, w, best);
    share = __shfl_sync(0xffffffffu, share, best);
    gaps = __shfl_sync(0xffffffffu, gaps, best);
    extra = gaps ? 0 : (int)__shfl_sync(0xffffffffu, ahead, best);
  }
  const int mates = warp / w, wi = warp - mates * w, team = mates * gridDim.x + blockIdx.x;
  int pos = team * share;
  auto team_sync = [&] {
    if (w == 1) __syncwarp();
    else group_sync(1 + mates, 32 * w);
  };
  // A unit's length in the line: nothing of nothing; where there are gaps, its blocks rounded up to whole shares (by a reciprocal that is never
  // too small and too large by less than one share, which is put right).
  const float per_share = __fdividef(1.f + 1e-6f, (float)share);
  auto length = [&](int blocks) {
    if (!gaps) return blocks == 0 ? 0 : blocks + extra;
    const int full = (int)((float)(blocks - 1) * per_share);
    return blocks == 0 ? 0 : (full * share <= blocks - 1 ? full + 1 : full) * share;
  };

  // The sequence in which the share begins, and where its units begin in the line.
  int b = 0, first = 0;
#pragma unroll 1
  for (;; b += 32) {
    if (b >= n_seqs) return;  // (behind the line's end)
    const int mine = b + lane < n_seqs ? length(k4_blocks<KT>(A, k4_len(A, A.seq_len[b + lane]))) * per_seq : 0;
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += x;
    }
    const uint32_t behind = __ballot_sync(0xffffffffu, pos < first + sum);
    if (behind) {
      const int at = __ffs(behind) - 1;
      b += at;
      first += __shfl_sync(0xffffffffu, sum - mine, at);
      break;
    }
    first += __shfl_sync(0xffffffffu, sum, 31);
  }
  const int end = pos + share;  // (or where the line ends)

  const int tok0 = (g & 1) ? 7 - (g >> 1) : g >> 1;   // row g of a product of keys; row g + 8 is 8 tokens further
  const uint64_t once = l2_evict_first();  // (pages pass through L2 without driving the kernel's own code out of it)
  int stage = 0;
  uint32_t parity = 0;
  bool dead = false;

  while (pos < end) {
    int len = k4_len(A, A.seq_len[b]), blocks = k4_blocks<KT>(A, len);
    while (pos >= first + length(blocks) * per_seq) {
      first += length(blocks) * per_seq;
      if (++b >= n_seqs) return;
      len = k4_len(A, A.seq_len[b]);
      blocks = k4_blocks<KT>(A, len);
    }
    // blocks from ... upto of a unit that begins in u0 of the line, with `extra` in front of its blocks
    const int line = length(blocks), unit = (unsigned)(pos - first) / (unsigned)line, u0 = first + unit * line, from_block = max(pos - u0 - extra, 0);
    const int left = min(end - u0 - extra, blocks) - from_block, seg = min(left, K4_RUN * w);  // (of the share, of this run)
    pos = seg < left ? u0 + extra + from_block + seg : min(u0 + line, end);
    if (left <= 0) continue;
    const int h = A.by_row_tiles(unit), row0 = (unit - h * A.row_tiles) * S::ROWS, rows = min(S::ROWS, A.q_len * A.group - row0);
    const int n = dead ? 0 : (unsigned)(seg + w - 1 - wi) / (unsigned)w;
    const int block0 = k4_first<KT>(A, len) + from_block + wi;

    // queries: the lane's columns of the operand are components 8 (4 j + t) ... of row g
    uint4 raw[N8][KW];
#pragma unroll
    for (int x = 0; x < N8; ++x) {
      const int r = row0 + (COLS ? g / NG : 8 * x + g), i = A.by_group(r);
      const uint16_t* src_q = A.q + ((long long)b * A.q_len + i) * A.q_stride + (long long)(h * A.group + r - i * A.group) * D + 8 * t;
#pragma unroll
      for (int j = 0; j < KW; ++j) {
        raw[x][j] = make_uint4(0, 0, 0, 0);
        if (r < row0 + rows) raw[x][j] = ldg128(src_q + 32 * j);
      }
    }

    // pages of 32 of this warp's blocks at a time, one to a lane, the next ones already asked for
    const int32_t* table = A.p.table + (long long)b * A.p.table_stride;
    int id[KT], id_next[KT];
    auto ask = [&](int j, int (&to)[KT]) {
#pragma unroll
      for (int i = 0; i < KT; ++i) {
        const int tile = (block0 + (j + lane) * w) * KT + i;
        to[i] = j + lane < n && tile * 16 < len ? table[A.by_page(tile)] : -1;
      }
    };
    ask(0, id);
    ask(32, id_next);
    uint32_t good[KT], skip = 0;  // (skip: KT bits by stage, tiles without a page; kept once there is one)
    bool patchy = false, joined = false;
    const uint8_t* src[KT];
    auto settle = [&](int j) {  // turns the asked numbers into addresses for blocks j ... j + 31
      bool all = true;
#pragma unroll
      for (int i = 0; i < KT; ++i) {
        const int tile = (block0 + (j + lane) * w) * KT + i;
        const bool none = i && tile * 16 >= len;  // (behind the sequence's end: what nobody sees may be the tile before)
        if (none) src[i] = src[0];
        const bool ok = none || (id[i] >= 0 && id[i] < A.p.n_pages);
        if (!ok && j + lane < n && tile * 16 < len) set_status(A.p.status, ST_BAD_INDEX);
        all &= ok || j + lane >= n;
        good[i] = __ballot_sync(0xffffffffu, none ? good[0] >> lane & 1 : ok);
        if (!none) src[i] = A.p.pages + (id[i] * A.p.page_stride + h * A.p.head_stride + (long long)(tile - A.by_page(tile) * (A.p.page >> 4)) * S::TILE);
      }
      joined = KT == 2 && all && src[KT - 1] == src[0] + S::TILE;  // (the lane's tiles side by side: one copy)
      patchy |= !__all_sync(0xffffffffu, all);
    };
    auto bulk = [&](int tile, const uint8_t* from, uint32_t bytes, uint32_t to) {
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(saddr(ring + tile * S::TILE)),
                   "l"(from), "r"(bytes), "r"(to), "l"(once) : "memory");
    };
    auto copy = [&](int j, int to) {
      uint32_t here = (1u << KT) - 1;
      if (patchy) {
        here = 0;
#pragma unroll
        for (int i = 0; i < KT; ++i) here |= (good[i] >> (j & 31) & 1) << i;
        skip = (skip & ~(((1u << KT) - 1) << (to * KT))) | (here ^ ((1u << KT) - 1)) << (to * KT);
      }
      if (lane == (j & 31)) {
        mb_expect(bar + 8 * to, __popc(here) * S::TILE);
        if (joined) bulk(to * KT, src[0], KT * S::TILE, bar + 8 * to);
        else {
#pragma unroll
          for (int i = 0; i < KT; ++i)
            if (here >> i & 1) bulk(to * KT + i, src[i], S::TILE, bar + 8 * to);
        }
      }
    };
    settle(0);
    {
      int to = stage;
#pragma unroll 1
      for (int j = 0; j < min(n, ST); ++j) {
        copy(j, to);
        to = to + 1 == ST ? 0 : to + 1;
      }
    }

    // Everything below is kept for the lane's two rows: 2 t and 2 t + 1, or g and g + 8 (or the columns 2 t and 2 t + 1 of one row).
    uint32_t qf[S::Q_SHARED ? 1 : N8][KW][4];
    // (E: factors of scales, of the groups, or of the lane's columns)
    float qs[NS][2], cn[2], M[2] = {-3e38f, -3e38f}, l[2] = {0.f, 0.f}, E[NV], zs[NS][2], cs[NS][4], o[NW][2][2][N8][4];
#pragma unroll
    for (int k = 0; k < NV; ++k) E[k] = NG > 1 ? K4_FACTOR : 1.f;
#pragma unroll
    for (int e = 0; e < 4 * NS; ++e) { cs[e / 4][e % 4] = 0.f; zs[e / 4][e % 2] = 0.f; }
#pragma unroll
    for (int e = 0; e < 16 * N8 * NW; ++e) o[e / (16 * N8)][e / (8 * N8) % 2][e / (4 * N8) % 2][e / 4 % N8][e % 4] = 0.f;
#pragma unroll
    for (int x = 0; x < N8; ++x) {
      float top = 0.f, part[NS];
#pragma unroll
      for (int j = 0; j < KW; ++j) {
        const uint32_t u[4] = {raw[x][j].x, raw[x][j].y, raw[x][j].z, raw[x][j].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 f = both_halves<WD>(u[e]);
          top = max3(top, fabsf(f.x), fabsf(f.y));
        }
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // the largest component of a row lies in [2^14, 2^15)
      const int ex = min(max((int)(__float_as_uint(top) >> 23) - 127, -100), 127);
      const float up = __uint_as_float((uint32_t)(14 - ex + 127) << 23), up16 = up * 0.0625f;
#pragma unroll
      for (int k = 0; k < NS; ++k) part[k] = 0.f;
#pragma unroll
      for (int j = 0; j < KW; ++j) {
        const uint32_t u[4] = {raw[x][j].x, raw[x][j].y, raw[x][j].z, raw[x][j].w};
        const int k = COLS ? 0 : 32 * j / G;
        const bool here = !COLS || 32 * j / G == g % NG;  // (a column without the components holds zeros)
        float2 f[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f[e] = both_halves<WD>(u[e]);
          if (!here) f[e] = make_float2(0.f, 0.f);
          part[k] = fmaf(f[e].x, up, fmaf(f[e].y, up, part[k]));
        }
        const uint4 q = make_uint4(halves(f[0].x * up, f[2].x * up), halves(f[0].y * up16, f[2].y * up16), halves(f[1].x * up, f[3].x * up),
                                   halves(f[1].y * up16, f[3].y * up16));
        if constexpr (S::Q_SHARED) *reinterpret_cast<uint4*>(q_shared + (x * KW + j) * 512) = q;
        else { qf[x][j][0] = q.x; qf[x][j][1] = q.y; qf[x][j][2] = q.z; qf[x][j][3] = q.w; }
      }
      const float c = fmaxf(A.scale_log2 * 4194304.f * __uint_as_float((uint32_t)(ex - 14 + 127) << 23), 1e-37f);  // (a masked score times it stays -inf)
      if (!(c < INFINITY)) part[0] = __int_as_float(0x7fffffff);
      if (WIDE) cn[x] = c;
      else { cn[0] = __shfl_sync(0xffffffffu, c, 8 * t); cn[1] = __shfl_sync(0xffffffffu, c, 8 * t + 4); }
#pragma unroll
      for (int k = 0; k < NS; ++k) {
        const float f = quad_sum(part[k]) * 2.384185791015625e-7f;  // 2^-22
        if (WIDE) qs[k][x] = f;
        else { qs[k][0] = __shfl_sync(0xffffffffu, f, 8 * t); qs[k][1] = __shfl_sync(0xffffffffu, f, 8 * t + 4); }
      }
    }
    // Blocks that all rows see all of: from `plain` on, `plains` of them.
    int plain, plains;
    {
      const int first_row = len - A.q_len + A.by_group(row0), last_row = len - A.q_len + A.by_group(row0 + rows - 1);
      const int upto = max(first_row + 1, 0) / (16 * KT);                                     // (blocks below it end at the first row or before)
      const int since = (int)((unsigned)max(max(last_row, 0) - A.window + 16 * KT, 0) / (16 * KT));  // (its first key and all behind are seen by the last row)
      plain = (unsigned)max(since - block0 + w - 1, 0) / (unsigned)w;
      plains = max((int)((unsigned)max(upto - block0 + w - 1, 0) / (unsigned)w) - plain, 0);
    }

#pragma unroll 1
    for (int j = 0; j < n; ++j) {
      bool here = mb_try(bar + 8 * stage, parity);
      if (!__all_sync(0xffffffffu, here)) {
        const long long began = clock64();
        do {
          if (!here) here = mb_try(bar + 8 * stage, parity);
          dead = __any_sync(0xffffffffu, !here && clock64() - began > K4_SPIN_CLOCKS);
        } while (!dead && !__all_sync(0xffffffffu, here));
        if (dead) {  // the copies still on their way get as long again to land
          set_status(A.p.status, ST_TIMEOUT);
          if (lane == 0) atomicOr(s_dead, 1 << warp);
          while (clock64() - began < 2 * K4_SPIN_CLOCKS) {}
          break;
        }
      }
      {
        const uint8_t* tile = ring + stage * KT * S::TILE;
        const bool edge = (unsigned)(j - plain) >= (unsigned)plains || patchy;

        // Scores.  NK keys of a tile are the lane's: tok0 and tok0 + 8, or t, 7 - t, 8 + t, 15 - t; score e is of row_of(e), key_of(e).
        constexpr int NK = 2 * N8, NX = NR * NK;
        auto row_of = [](int e) { return COLS ? 0 : WIDE ? e / 2 % 2 : e % 2; };
        auto key_of = [](int e) { return COLS ? e : WIDE ? e / 4 * 2 + e % 2 : e / 2; };
        auto token_of = [&](int k) { return WIDE ? (k & 2) * 4 + (k & 1 ? 7 - t : t) : tok0 + 8 * k; };
        const int my_group = COLS ? 2 * t % NG * 4 : 0;
        float x[KT][NX];
        {
          uint32_t ka[KT][KW], kb[KT][KW], meta[KT][NK][NV];
          constexpr int n4 = D == 64 ? 2 : 4;
#pragma unroll
          for (int z = 0; z < KT; ++z) {
            const uint8_t* mine = tile + z * S::TILE;
#pragma unroll
            for (int half = 0; half < KW / n4; ++half) {
              const int off = ((D == 256 ? half ^ (tok0 & 1) : 0) * 4 + t) * n4 * 4;
              uint32_t a[n4], c[n4];
              lds_words<n4>(mine + tok0 * (D / 2) + off, a);
              lds_words<n4>(mine + (tok0 + 8) * (D / 2) + off, c);
#pragma unroll
              for (int i = 0; i < n4; ++i) { ka[z][half * n4 + i] = a[i]; kb[z][half * n4 + i] = c[i]; }
            }
#pragma unroll
            for (int k = 0; k < NK; ++k) lds_words<NV>(mine + 16 * D + token_of(k) * 4 * NG + my_group, meta[z][k]);
          }
#pragma unroll
          for (int k = 0; k < NS; ++k) {
            constexpr int part = KW / NS;  // (words of a code row for one sum)
            float acc[KT][N8][4];
#pragma unroll
            for (int i = k * part; i < (k + 1) * part; ++i) {
              uint32_t q[N8][4];
#pragma unroll
              for (int y = 0; y < N8; ++y) {
                if constexpr (S::Q_SHARED) lds_words<4>(q_shared + (y * KW + i) * 512, q[y]);
                else {
#pragma unroll
                  for (int e = 0; e < 4; ++e) q[y][e] = qf[y][i][e];
                }
              }
#pragma unroll
              for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int z = 0; z < KT; ++z) {
                  const uint32_t a = s ? ka[z][i] >> 6 : ka[z][i] << 2, c = s ? kb[z][i] >> 6 : kb[z][i] << 2;
                  const uint32_t a0 = a & 0x003c003cu, a1 = a & 0x03c003c0u, c0 = c & 0x003c003cu, c1 = c & 0x03c003c0u;
                  const bool first = i == k * part && s == 0;
                  if constexpr (WIDE) {
                    mma_f16(acc[z][0], q[0][2 * s], q[1][2 * s], q[0][2 * s + 1], q[1][2 * s + 1], a0, a1, first);
                    mma_f16(acc[z][1], q[0][2 * s], q[1][2 * s], q[0][2 * s + 1], q[1][2 * s + 1], c0, c1, first);
                  } else mma_f16(acc[z][0], a0, c0, a1, c1, q[0][2 * s], q[0][2 * s + 1], first);
                }
            }
#pragma unroll
            for (int z = 0; z < KT; ++z) {
              if constexpr (COLS) {
#pragma unroll
                for (int i = 0; i < NK; ++i) {
                  const float2 m0 = both_halves<WD>(meta[z][i][0]), m1 = both_halves<WD>(meta[z][i][1]);
                  float v = fmaf(m0.x, acc[z][0][2 * i], m0.y * qs[0][0]) + fmaf(m1.x, acc[z][0][2 * i + 1], m1.y * qs[0][1]);
                  if (NG >= 4) v += __shfl_xor_sync(0xffffffffu, v, 1);
                  if (NG >= 8) v += __shfl_xor_sync(0xffffffffu, v, 2);
                  x[z][i] = v;
                }
              } else {
                float2 m[NK];
#pragma unroll
                for (int i = 0; i < NK; ++i) m[i] = both_halves<WD>(meta[z][i][k]);
#pragma unroll
                for (int e = 0; e < NX; ++e) {
                  const float2 sz = m[key_of(e)];
                  const float zero = k ? fmaf(sz.y, qs[k][row_of(e)], x[z][e]) : sz.y * qs[k][row_of(e)];
                  x[z][e] = fmaf(sz.x, acc[z][e / 4][e % 4], zero);
                }
              }
            }
          }
        }
        // scales and zeros of the values of the same tokens, as scales and middles
        float2 va[KT][NK][NV];
#pragma unroll
        for (int z = 0; z < KT; ++z)
#pragma unroll
          for (int i = 0; i < NK; ++i) {
            uint32_t meta[NV];
            lds_words<NV>(tile + z * S::TILE + 16 * D + 64 * NG + token_of(i) * 4 * NG + my_group, meta);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
              va[z][i][k] = both_halves<WD>(meta[k]);
              va[z][i][k].y = fmaf(va[z][i][k].x, 8.f, va[z][i][k].y);  // (the middle of what the codes stand for)
            }
          }
        if (edge) {
          const uint32_t gone = skip >> (stage * KT);
          const int pos0 = (block0 + j * w) * 16 * KT;
          // Tokens that nobody sees may hold anything, and one that some rows see may hold NaN: neither must meet a weight of zero.
          int hi[2], lo[2];
#pragma unroll
          for (int e = 0; e < NR; ++e) {
            const int r = COLS ? 2 * t / NG : WIDE ? 8 * e + g : 2 * t + e;
            hi[e] = r < rows ? len - A.q_len + A.by_group(row0 + r) : -1;
            lo[e] = max(hi[e], -1) - A.window;
          }
#pragma unroll
          for (int z = 0; z < KT; ++z)
#pragma unroll
            for (int i = 0; i < NK; ++i) {
              const int at = pos0 + 16 * z + token_of(i);
              bool on[2] = {false, false}, fine[NV];
#pragma unroll
              for (int e = 0; e < NR; ++e) on[e] = !(gone >> z & 1) && at <= hi[e] && at > lo[e];
#pragma unroll
              for (int e = 0; e < NX; ++e)
                if (key_of(e) == i && !on[row_of(e)]) x[z][e] = -INFINITY;
              // (the lanes that share the key: those of the same t, or of the same g)
              const bool any = __ballot_sync(0xffffffffu, on[0] || on[1]) & (WIDE ? 0x11111111u << t : 15u << (lane & 28));
#pragma unroll
              for (int k = 0; k < NV; ++k) {
                fine[k] = fabsf(va[z][i][k].x) + fabsf(va[z][i][k].y) < INFINITY;
#pragma unroll
                for (int e = 0; e < NR; ++e)
                  if (on[e] && !fine[k]) zs[COLS ? 0 : k][COLS ? k : e] = __int_as_float(0x7fffffff);
                if (!any || !fine[k]) va[z][i][k] = make_float2(0.f, 0.f);
              }
            }
        }
        // Scales of a head's groups may differ by any power: each counts times a factor E, a power of two that brings the largest of a group so far
        // near 1 (none where a head has one group), which is taken off in the end.
        // Weights relative to M, which moves only when the weights times their scales leave what fp16 holds, or times their middles 2^104 (bf16
        // alone can: sums of 2^24 of them stay in fp32's range).  (Their sum tells: none of them is negative, and one that is NaN may hide
        // nothing; `least` keeps weights of scales of zero in range.)
        constexpr float least = WD == WD_BF16 ? 0x1p-90f : 0x1p-60f;
        auto scaled = [&](int z, int i, int k) { return NG > 1 ? va[z][i][k].x * E[k] : va[z][i][k].x; };
        auto size_of = [&](int z, int i, int k, float and_) {
          const float2 v = va[z][i][k];
          if (WD == WD_BF16) and_ = fmaf(fabsf(v.y), 0x1p-90f, and_);
          return NG > 1 ? fmaf(v.x, E[k], and_) : v.x + and_;
        };
        float p[KT][NX], most[2] = {0.f, 0.f};
#pragma unroll
        for (int z = 0; z < KT; ++z) {
          float all[NK];
#pragma unroll
          for (int i = 0; i < NK; ++i) {
            all[i] = least;
#pragma unroll
            for (int k = 0; k < NV; ++k) all[i] = size_of(z, i, k, all[i]);
          }
#pragma unroll
          for (int e = 0; e < NX; ++e) {
            p[z][e] = ex2(fmaf(x[z][e], cn[row_of(e)], -M[row_of(e)]));
            most[e % 2] = fmaf(p[z][e], all[key_of(e)], most[e % 2]);
          }
        }
        if (__any_sync(0xffffffffu, !(most[0] + most[1] <= 16384.f))) {
          // (Scores so large that their last place counts are rounded before M is, and no weight is above what M allows: a row's largest
          // score then has a weight that is neither 0 nor infinite.)
          float m[2] = {-INFINITY, -INFINITY}, f[2], big[KT][NK], h[NV];
#pragma unroll
          for (int k = 0; k < NV; ++k) {
            h[k] = 1.f;
            if constexpr (NG > 1) {
              float s = 0.f;
#pragma unroll
              for (int z = 0; z < KT; ++z)
#pragma unroll
                for (int i = 0; i < NK; ++i) s = fmaxf(s, va[z][i][k].x);
              s = WIDE ? quad_max(s) : rows_max(s);
              if (s * E[k] > 64.f) {
                const float to = fmaxf(__uint_as_float((254u - (__float_as_uint(s) >> 23)) << 23), K4_LEAST_FACTOR);
                h[k] = __fdividef(to, E[k]);
                E[k] = to;
              }
            }
          }
#pragma unroll
          for (int z = 0; z < KT; ++z) {
#pragma unroll
            for (int i = 0; i < NK; ++i) {
              big[z][i] = least;
#pragma unroll
              for (int k = 0; k < NV; ++k) big[z][i] = fmaxf(big[z][i], size_of(z, i, k, 0.f));
              if (COLS && NG >= 4) big[z][i] = fmaxf(big[z][i], __shfl_xor_sync(0xffffffffu, big[z][i], 1));  // (one weight for all groups)
              if (COLS && NG >= 8) big[z][i] = fmaxf(big[z][i], __shfl_xor_sync(0xffffffffu, big[z][i], 2));
              big[z][i] = __log2f(big[z][i]) - 4.f;
            }
#pragma unroll
            for (int e = 0; e < NX; ++e) m[row_of(e)] = fmaxf(m[row_of(e)], __fmul_rn(x[z][e], cn[row_of(e)]) + big[z][key_of(e)]);
          }
#pragma unroll
          for (int e = 0; e < NR; ++e) {
            const float to = fmaxf(M[e], WIDE ? quad_max(m[e]) : rows_max(m[e]));
            f[e] = ex2(M[e] - to);
            M[e] = to;
            l[e] *= f[e];
          }
          if (COLS) f[1] = f[0];
#pragma unroll
          for (int k = 0; k < NS; ++k) {
#pragma unroll
            for (int e = 0; e < 2; ++e) zs[k][e] *= f[e];
#pragma unroll
            for (int e = 0; e < 4; ++e) cs[k][e] *= f[WIDE ? e / 2 : e % 2] * h[COLS ? e % 2 : k];
          }
#pragma unroll
          for (int e = 0; e < 16 * N8 * NW; ++e)
            o[e / (16 * N8)][e / (8 * N8) % 2][e / (4 * N8) % 2][e / 4 % N8][e % 4] *= f[WIDE ? e / 2 % 2 : e % 2] * h[COLS ? e % 2 : 32 * (e / (8 * N8)) / G];
#pragma unroll
          for (int z = 0; z < KT; ++z)
#pragma unroll
            for (int e = 0; e < NX; ++e) {
              const float y = __fsub_rn(__fmul_rn(x[z][e], cn[row_of(e)]), M[row_of(e)]), room = -big[z][key_of(e)];
              p[z][e] = ex2(y > room ? room : y);  // (NaN stays)
            }
        }
        // Weights times scales, rounded to fp16 for the product with the codes.  The codes count from the middle of their range, 8: the
        // rounding then weighs s |u - 8|, about a value's own size.  8 sum(p s) is taken off with the rounded weights (a product with
        // ones), and added back, unrounded, with the zeros.
        uint32_t pf[KT][NS][NK];
#pragma unroll
        for (int z = 0; z < KT; ++z) {
#pragma unroll
          for (int e = 0; e < NX; ++e) l[row_of(e)] += p[z][e];
#pragma unroll
          for (int k = 0; k < NS; ++k) {
            if constexpr (COLS) {
#pragma unroll
              for (int i = 0; i < NK; ++i) {
                const float2 a = va[z][i][0], c = va[z][i][1];
                zs[0][0] = fmaf(p[z][i], a.y, zs[0][0]);
                zs[0][1] = fmaf(p[z][i], c.y, zs[0][1]);
                pf[z][0][i] = transpose8(halves(p[z][i] * scaled(z, i, 0), p[z][i] * scaled(z, i, 1)));
              }
            } else {
#pragma unroll
              for (int e = 0; e < NX; ++e) zs[k][row_of(e)] = fmaf(p[z][e], va[z][key_of(e)][k].y, zs[k][row_of(e)]);
#pragma unroll
              for (int e = 0; e < NX; e += 2) {
                const uint32_t two = halves(p[z][e] * scaled(z, key_of(e), k), p[z][e + 1] * scaled(z, key_of(e + 1), k));
                pf[z][k][e / 2] = WIDE ? two : transpose8(two);
              }
            }
            if constexpr (WIDE) mma_f16(cs[k], pf[z][k][0], pf[z][k][1], pf[z][k][2], pf[z][k][3], 0x3c003c00u, 0x3c003c00u);
            else mma_f16(cs[k], 0x3c003c00u, 0u, 0x3c003c00u, 0u, pf[z][k][0], pf[z][k][1]);
          }
        }
        // Values, summed over the tokens t, 7 - t, 8 + t, 15 - t of the lane.  Its words hold components of g.
#pragma unroll
        for (int z = 0; z < KT; ++z) {
          const uint8_t* base = tile + z * S::TILE + 16 * (D / 2);
          uint32_t v[4][NW];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int row = (i & 2) * 4 + (i & 1 ? 7 - t : t);
            lds_words<NW>(base + row * (D / 2) + value_word<D>(g, 0, row) * 4, v[i]);
          }
#pragma unroll
          for (int ws = 0; ws < NW; ++ws)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const uint32_t a = __byte_perm(v[0][ws], v[1][ws], half ? 0x7632 : 0x5410), c = __byte_perm(v[2][ws], v[3][ws], half ? 0x7632 : 0x5410);
#pragma unroll
              for (int s = 0; s < 2; ++s) {
                const int k = COLS ? 0 : (64 * ws + 32 * half) / G;
                const uint32_t d = s ? a >> 6 : a << 2, f = s ? c >> 6 : c << 2;
                const uint32_t d0 = d & 0x003c003cu, d1 = d & 0x03c003c0u, f0 = f & 0x003c003cu, f1 = f & 0x03c003c0u;
                if constexpr (WIDE) {
                  mma_f16(o[ws][half][s][0], pf[z][k][0], pf[z][k][1], pf[z][k][2], pf[z][k][3], d0, f0);
                  mma_f16(o[ws][half][s][1], pf[z][k][0], pf[z][k][1], pf[z][k][2], pf[z][k][3], d1, f1);
                } else mma_f16(o[ws][half][s][0], d0, d1, f0, f1, pf[z][k][0], pf[z][k][1]);
              }
            }
        }
      }
      if (j % K4_MIDDLE == K4_MIDDLE - 1) {
#pragma unroll
        for (int e = 0; e < 16 * N8 * NW; ++e) {
          const int at = e / (8 * N8), s = e / (4 * N8) % 2, c = e % 4;
          const bool high = WIDE ? e / 4 % 2 : c >= 2;  // (codes at bit 6)
          float& sum = o[at / 2][at % 2][s][e / 4 % N8][c];
          sum = fmaf(high ? -0x1p-15f : -0x1p-19f, cs[COLS ? 0 : 32 * at / G][WIDE ? c : c % 2], sum);
        }
#pragma unroll
        for (int e = 0; e < 4 * NS; ++e) cs[e / 4][e % 4] = 0.f;
      }
      __syncwarp();
      if (j + ST < n) {
        if (((j + ST) & 31) == 0) {
#pragma unroll
          for (int i = 0; i < KT; ++i) id[i] = id_next[i];
          ask(j + ST + 32, id_next);
          settle(j + ST);
        }
        copy(j + ST, stage);
      }
      if (++stage == ST) { stage = 0; parity ^= 1; }
    }

    // the warp's sums, in shared memory
    {
      float* piece = reinterpret_cast<float*>(ring);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float sum_l = WIDE ? quad_sum(l[e]) : rows_sum(l[COLS ? 0 : e]);
        float zero[NS], one[NS];
#pragma unroll
        for (int k = 0; k < NS; ++k) {
          one[k] = __fdividef(1.f, E[COLS ? e : k]);
          zero[k] = fmaf(-8.f * one[k], cs[k][WIDE ? 2 * e : e], WIDE ? quad_sum(zs[k][e]) : rows_sum(zs[k][e]));
        }
        float* line = piece + (COLS ? (2 * t + e) / NG : WIDE ? 8 * e + g : 2 * t + e) * S::LINE;
        // four components side by side: of g, or, twice, of 2 t and 2 t + 1 (of a column that stands for one group, that group's)
#pragma unroll
        for (int i = 0; i < 2 * NW * N8; ++i) {
          const int at = i / N8, c = WIDE ? 2 * e + i % 2 : e;
          if (COLS && (2 * t + e) % NG != 32 * at / G) continue;
          const float zz = zero[COLS ? 0 : 32 * at / G], low = 4194304.f * one[COLS ? 0 : 32 * at / G], high = 262144.f * one[COLS ? 0 : 32 * at / G];
          const auto& a = o[at / 2][at % 2];
          const float first = a[0][0][c], second = WIDE ? a[0][N8 - 1][c] : a[0][0][c + 2], third = a[1][0][c], last = WIDE ? a[1][N8 - 1][c] : a[1][0][c + 2];
          *reinterpret_cast<float4*>(line + 32 * at + 4 * (WIDE ? 2 * t + i % 2 : g)) =
              make_float4(fmaf(first, low, zz), fmaf(second, high, zz), fmaf(third, low, zz), fmaf(last, high, zz));
        }
        if (WIDE ? t == 0 : g == 0 && (!COLS || (2 * t + e) % NG == 0)) *reinterpret_cast<float2*>(line + D) = make_float2(M[COLS ? 0 : e], sum_l);
      }
    }
    team_sync();
    // The team's pieces are added up, to the output or to the workspace; there, the team that comes last fetches the unit's pieces, as many as
    // its place holds at a time, and adds them up by the same code (which the SM has at hand by now; code of its own is cold).
    const int i0 = (u0 + extra) / share, i1 = (u0 + extra + blocks - 1) / share;  // the unit's teams
    const int items = rows * (D / 4), threads = 32 * w, me = wi * 32 + lane, room = w * S::RING / S::PIECE;
    // Of several runs, all but the last leave their sums in the workspace, where the next finds them; M and the sum of weights stand in two places by turns
    // (other threads may still read the last ones), the last time in the first.
    const int runs = left == seg ? 0 : (unsigned)(left - seg + K4_RUN * w - 1) / (unsigned)(K4_RUN * w), ml_to = D + 2 * (runs & 1), ml_last = D + 2 * (~runs & 1);
    bool more = from_block > max(team * share - u0 - extra, 0);
    const bool whole = from_block + left == blocks && max(team * share - u0 - extra, 0) == 0;
    float* place = reinterpret_cast<float*>(smem + (warp - wi) * S::RING);
    const float* from = place;                                                                // what is added up: `count` pieces,
    float* kept = A.part + (long long)(2 * team + (team == i0)) * (S::PIECE / 4);
    float* to = kept;                                                                         // and where it goes
    int count = w, stride = S::RING / 4, next = whole && runs == 0 ? i1 + 1 : -1;  // (next: the team whose piece is fetched next)
#pragma unroll 1
    for (;;) {
      const bool done = next > i1;
#pragma unroll 1
      for (int x = me; x < items; x += threads) {
        const int r = x / (D / 4), c = x % (D / 4) * 4;
        float m = -INFINITY, sum_l = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (more) {
          const float2 ml = __ldcg(reinterpret_cast<const float2*>(kept + r * S::LINE + ml_last));
          m = ml.x;
          sum_l = ml.y;
          v = __ldcg(reinterpret_cast<const float4*>(kept + r * S::LINE + c));
        }
        const float* line = from + r * S::LINE;
#pragma unroll 2
        for (int i = 0; i < count; ++i, line += stride) {
          const float4 y = *reinterpret_cast<const float4*>(line + c);
          const float2 ml = *reinterpret_cast<const float2*>(line + D);
          k4_add(m, sum_l, v, ml.x, ml.y, y);
        }
        if (*s_dead & ((1 << w) - 1) << (warp - wi)) sum_l = __int_as_float(0x7fffffff);
        if (!done) {
          *reinterpret_cast<float4*>(to + r * S::LINE + c) = v;
          if (c == 0) *reinterpret_cast<float2*>(to + r * S::LINE + (to == kept ? ml_to : D)) = make_float2(m, sum_l);
          continue;
        }
        const int i = A.by_group(row0 + r), hd = h * A.group + (row0 + r - i * A.group);
        const long long tk = (long long)b * A.q_len + i;
        const float f = sum_l == 0.f ? 0.f : __fdividef(1.f, sum_l);
        uint16_t* dst = A.out + tk * A.out_stride + (long long)hd * D + c;
        const uint2 word = make_uint2(pack2<WD>(v.x * f, v.y * f), pack2<WD>(v.z * f, v.w * f));
        if (A.out_vec) *reinterpret_cast<uint2*>(dst) = word;
        else { dst[0] = (uint16_t)word.x; dst[1] = (uint16_t)(word.x >> 16); dst[2] = (uint16_t)word.y; dst[3] = (uint16_t)(word.y >> 16); }
        if (c == 0 && A.lse) A.lse[tk * A.heads + hd] = sum_l == 0.f ? -INFINITY : (m + __log2f(sum_l)) * LN2;
      }
      if (done || runs) break;
      more = false;
      team_sync();
      int have = 1;
      if (next < 0) {
        if (me == 0) {  // (the barrier orders the team's stores before this thread's fence)
          int32_t* arrived = A.arrived + ((long long)b * per_seq + unit);
          __threadfence();
          const int last = atomicAdd(arrived, 1) == i1 - i0;
          if (last) *arrived = 0;
          __threadfence();
          s_last[warp] = last;
        }
        team_sync();
        if (!s_last[warp - wi]) break;
        next = i0;
        have = 0;
        to = place;
      }
      // What was added up so far stands at one end of the place; pieces follow, and the next sum goes to the other end.
      from = to;
      stride = to == place ? S::PIECE / 4 : -(S::PIECE / 4);
      to = to == place ? place + (room - 1) * (S::PIECE / 4) : place;
      const int fetch = min(i1 + 1 - next, room - 1 - have);
#pragma unroll 1
      for (int i = wi; i < fetch; i += w) {
        const int at = next + i;
        const float4* src_p = reinterpret_cast<const float4*>(A.part + (long long)(2 * at + (at == i0)) * (S::PIECE / 4));
        float4* dst_p = reinterpret_cast<float4*>(const_cast<float*>(from) + (have + i) * stride);
#pragma unroll 1
        for (int x = lane; x < S::PIECE / 16; x += 9 * 32) {
          float4 y[9];
#pragma unroll
          for (int k = 0; k < 9; ++k)
            if (x + 32 * k < S::PIECE / 16) y[k] = __ldcg(src_p + x + 32 * k);
#pragma unroll
          for (int k = 0; k < 9; ++k)
            if (x + 32 * k < S::PIECE / 16) dst_p[x + 32 * k] = y[k];
        }
      }
      next += fetch;
      count = have + fetch;
      team_sync();
    }
    team_sync();
    fence_async_shared();  // (the next copies land where the piece was)
  }
}

}  // namespace ls
