// Attention over the 4-bit paged cache: queries of a few tokens per sequence against all of its keys.
//
// With u the codes and (s, z) scale and zero of a group, key j and value j are s_j u_j + z_j, so that (sums over groups left out)
//   score_j = scale (s_j <q, u_j> + z_j sum(q)),   out = (sum_j p_j s_j u_j + sum_j p_j z_j) / sum_j p_j,   p_j = e^(score_j - M).
// Both products take the codes themselves: four bits in the mantissa of a 16-bit float with an exponent of zero are a subnormal
// number, u 2^-24 times their place, exact in the tensor cores, so a word of eight codes becomes four operand registers with a few
// shifts and logical instructions and no conversion.  The sums of a product are aligned to 2^-14, not to what the subnormal numbers come
// to, so a code at bit 0 loses what lies below 2^-14 of a unit: keys' codes stand at bits 2 and 6 (2^-16; the 2^-4 between the two goes
// into the query), those of values, whose sum is compared with 8 times that of the weights, all at bit 6 (2^-20).
// Queries are scaled to a power of two per row and are exact in fp16, whatever the cache's type.
#pragma once
#include "ls_attend.cuh"
#include "ls_kv4.cuh"
#include "ls_tmem.cuh"

namespace ls {

struct Attend4Args {
  Kv4Pages p;
  const uint16_t* q;   // [n_seqs * q_len][heads][dim], token stride q_stride
  uint16_t* out;
  float* lse;          // [n_seqs * q_len][heads] or NULL
  const int32_t* seq_len;
  float* part;         // pieces of rows: [2 * teams][rows of a unit][dim + 4]: sums of values, then M (log 2) and the sum of weights
  int32_t* arrived;    // [units], zero between calls: pieces that are written
  int64_t q_stride, out_stride;
  int32_t q_len, heads, group, window, row_tiles, q_vec, out_vec, bf16;
  float scale_log2;
};

constexpr long long K4_SPIN_CLOCKS = 4000000000LL;  // about two seconds

// Shapes of the kernel: D components a head, groups of G, NT times 8 rows of queries at once.
template <int D, int G, int NT>
struct K4Shape {
  static constexpr int WARPS = D * NT <= 128 ? 16 : 8;   // (128 registers a thread, or 255)
  static constexpr int THREADS = WARPS * 32;
  static constexpr int ROWS = 8 * NT;
  static constexpr int NG = D / G;
  static constexpr int TILE = kv4_tile(D, G);
  static constexpr int LINE = D + 4;                     // floats of a row's piece
  static constexpr int PIECE = ROWS * LINE * 4;
  static constexpr int FIT = (232448 - 1024 - THREADS * 8 - WARPS * 64) / (WARPS * TILE);
  static constexpr int STAGES = FIT < 8 ? FIT : 8;
  // a warp's ring of tiles; once it is empty, at a unit's end, the same place holds the warp's piece
  static constexpr int RING = (STAGES * TILE > PIECE ? STAGES * TILE : PIECE);
  static constexpr int SMEM = WARPS * (RING + 64) + THREADS * 8 + 1024;
  static_assert(STAGES >= 3 && SMEM <= 232448, "ring");
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t halves(float lo, float hi) { return pack2<WD_FP16>(lo, hi); }
__device__ __forceinline__ float2 meta_values(uint32_t m, bool bf16) {
  if (bf16) return make_float2(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
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

// What sequence b has to be read: its length, first tile and number of tiles.
struct K4Seq { int len, t0, tiles; };
__device__ __forceinline__ K4Seq k4_seq(const Attend4Args& A, int b, bool report) {
  int n = A.seq_len[b];
  const long long most = min((long long)A.p.table_width * A.p.page, (long long)MAX_POSITIONS);
  if (n < 0 || n > most) {
    if (report) set_status(A.p.status, ST_BAD_INDEX);
    n = n < 0 ? 0 : (int)most;
  }
  const int lo = A.window >= n ? 0 : max(0, n - A.window - A.q_len + 1);
  return {n, lo / 16, (n + 15) / 16 - lo / 16};
}

// Rows of a piece or of a joined unit: four components of one row to the output.
__device__ __forceinline__ void k4_put(const Attend4Args& A, int b, int h, int r, int D, int c, float4 o, float m, float l) {
  const int i = r / A.group, hd = h * A.group + (r - i * A.group);
  const long long t = (long long)b * A.q_len + i;
  const float f = l == 0.f ? 0.f : 1.f / l;
  uint16_t* dst = A.out + t * A.out_stride + (long long)hd * D + c;
  uint2 w;
  if (A.bf16) w = make_uint2(pack2<WD_BF16>(o.x * f, o.y * f), pack2<WD_BF16>(o.z * f, o.w * f));
  else w = make_uint2(pack2<WD_FP16>(o.x * f, o.y * f), pack2<WD_FP16>(o.z * f, o.w * f));
  if (A.out_vec) *reinterpret_cast<uint2*>(dst) = w;
  else { dst[0] = (uint16_t)w.x; dst[1] = (uint16_t)(w.x >> 16); dst[2] = (uint16_t)w.y; dst[3] = (uint16_t)(w.y >> 16); }
  if (c == 0 && A.lse) A.lse[t * A.heads + hd] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
}

// A unit is one sequence's tiles (16 keys each) for one key head and one row tile of its queries.  All units' tiles stand in one line,
// cut into equal shares; a share belongs to a team of 1, 2, 4 ... warps, which deal out its tiles among themselves.  A warp copies its
// tiles by itself (bulk copies into a ring of its own) and works alone until a unit's end; then the team adds up, and a unit that
// reaches over several teams is joined, in order, by whichever of them comes last.
template <int D, int G, int NT>
__global__ void __launch_bounds__(K4Shape<D, G, NT>::THREADS, 1) ls_kv4_attend_kernel(const Attend4Args A) {
  using S = K4Shape<D, G, NT>;
  constexpr int NG = S::NG, NW = D / 64, KW = D / 32, ST = S::STAGES;
  extern __shared__ __align__(128) uint8_t smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  uint8_t* ring = smem + warp * S::RING;
  float* piece = reinterpret_cast<float*>(ring);
  uint8_t* rest = smem + S::WARPS * S::RING;
  const uint32_t bar = saddr(rest + warp * 64);
  long long* s_before = reinterpret_cast<long long*>(rest + S::WARPS * 64);      // [THREADS]
  long long* s_warp = s_before + S::THREADS;                                      // [WARPS]
  int* s_units = reinterpret_cast<int*>(s_warp + S::WARPS);                       // [WARPS]
  int* s_last = s_units + S::WARPS;                                               // [WARPS]
  int* s_dead = s_last + S::WARPS;                                                // [WARPS]
  if (lane < ST) mb_init(bar + 8 * lane, 1);
  fence_async_shared();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // the line: a chunk of sequences to each thread
  const int per_seq = A.p.kv_heads * A.row_tiles, chunk = (A.p.n_seqs + S::THREADS - 1) / S::THREADS;
  long long mine = 0;
  int busy = 0;
  for (int b = tid * chunk; b < min(A.p.n_seqs, (tid + 1) * chunk); ++b) {
    const int n = k4_seq(A, b, blockIdx.x == 0).tiles;
    mine += (long long)n * per_seq;
    busy += n > 0;
  }
  long long sum = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long x = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += x;
  }
  busy = __reduce_add_sync(0xffffffffu, busy);
  if (lane == 31) { s_warp[warp] = sum; s_units[warp] = busy; }
  __syncthreads();
  long long total = 0, before = sum - mine;
  int seqs = 0;
  for (int i = 0; i < S::WARPS; ++i) {
    if (i < warp) before += s_warp[i];
    total += s_warp[i];
    seqs += s_units[i];
  }
  s_before[tid] = before;
  __syncthreads();
  // sequences without a key
  if (seqs < A.p.n_seqs) {
    for (int b = blockIdx.x; b < A.p.n_seqs; b += gridDim.x) {
      if (k4_seq(A, b, false).tiles) continue;
      const int rows = A.q_len * A.group;
      for (long long x = tid; x < (long long)A.p.kv_heads * rows * (D / 4); x += S::THREADS) {
        const int c = (int)(x % (D / 4)) * 4;
        const long long y = x / (D / 4);
        k4_put(A, b, (int)(y / rows), (int)(y % rows), D, c, make_float4(0.f, 0.f, 0.f, 0.f), 0.f, 0.f);
      }
    }
  }
  if (total == 0) return;

  // Teams: a whole CTA where units are long, single warps where they are short.
  int lw = S::WARPS == 16 ? 4 : 3;
  {
    const long long mean = total / ((long long)seqs * per_seq);
    const long long share1 = total / ((long long)gridDim.x * S::WARPS);
    while (lw > 0 && share1 >= 2 && mean < (16 << lw)) --lw;
  }
  const int w = 1 << lw, wi = warp & (w - 1), team = (warp >> lw) * gridDim.x + blockIdx.x;
  const long long teams = (long long)gridDim.x * (S::WARPS >> lw), share = max((total + teams - 1) / teams, (long long)w);
  long long pos = team * share;
  const long long end = min(total, pos + share);
  auto team_sync = [&] {
    if (lw == 0) __syncwarp();
    else group_sync(1 + (warp >> lw), 32 << lw);
  };

  // the sequence in which the share begins
  int b = 0;
  long long first = 0;  // where its units begin in the line
  if (pos < end) {
    int lo = 0, hi = S::THREADS - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (s_before[mid] <= pos) lo = mid;
      else hi = mid - 1;
    }
    b = lo * chunk;
    first = s_before[lo];
  }
  uint32_t phase = 0, flying = 0;  // bits by stage
  bool dead = false;
  const int tok0 = (g & 1) ? 7 - (g >> 1) : g >> 1;   // row g of a product of keys; row g + 8 is 8 tokens further
  const int tpp = A.p.page / 16;

  while (pos < end) {
    K4Seq sq = k4_seq(A, b, false);
    while (sq.tiles == 0 || pos >= first + (long long)sq.tiles * per_seq) {
      first += (long long)sq.tiles * per_seq;
      sq = k4_seq(A, ++b, false);
    }
    const int unit = (int)((pos - first) / sq.tiles), skip = (int)(pos - first - (long long)unit * sq.tiles);
    const int seg = (int)min((long long)(sq.tiles - skip), end - pos);
    const int h = unit / A.row_tiles, row0 = (unit - h * A.row_tiles) * S::ROWS, rows = min(S::ROWS, A.q_len * A.group - row0);
    const int n = seg > wi ? (seg - wi + w - 1) >> lw : 0;
    const int tile0 = sq.t0 + skip + wi;

    // pages of 32 of this warp's tiles at a time, one to a lane, the next ones already asked for
    const int32_t* table = A.p.table + (long long)b * A.p.table_stride;
    auto ask = [&](int j) { return j + lane < n ? table[(tile0 + (j + lane) * w) / tpp] : -1; };
    int id = ask(0), id_next = ask(32);
    uint32_t good = 0, good_before = 0;
    long long src = 0;
    auto settle = [&](int j) {  // turns the asked numbers into addresses for tiles j ... j + 31
      const bool ok = id >= 0 && id < A.p.n_pages;
      if (!ok && j + lane < n) set_status(A.p.status, ST_BAD_INDEX);
      good_before = good;
      good = __ballot_sync(0xffffffffu, ok);
      const int tile = tile0 + (j + lane) * w;
      src = id * A.p.page_stride + h * A.p.head_stride + (long long)(tile % tpp) * S::TILE;
    };
    auto copy = [&](int j, int stage) {
      if (j && (j & 31) == 0) { id = id_next; id_next = ask(j + 32); settle(j); }
      if (dead || !(good >> (j & 31) & 1)) return;
      flying |= 1u << stage;
      if (lane == (j & 31)) {
        mb_expect(bar + 8 * stage, S::TILE);
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(saddr(ring + stage * S::TILE)),
                     "l"(A.p.pages + src), "r"(S::TILE), "r"(bar + 8 * stage) : "memory");
      }
    };
    settle(0);
#pragma unroll 1
    for (int j = 0; j < min(n, ST); ++j) copy(j, j);

    // queries: the lane's columns of the operand are components 8 (4 j + t) ... of row g
    uint32_t qf[NT][KW][4];
    float qs[NT][NG][2], cn[NT][2], M[NT][2], l[NT][2], zs[NT][NG][2], cs[NT][NG][4], o[NT][NW][2][2][4];
    int at[NT][2];
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      const int r = row0 + 8 * x + g;
      float v[KW][8], top = 0.f, part[NG];
      const int i = r / A.group;
      const uint16_t* src_q = A.q + ((long long)b * A.q_len + i) * A.q_stride + (long long)(h * A.group + r - i * A.group) * D + 8 * t;
#pragma unroll
      for (int j = 0; j < KW; ++j) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[j][e] = 0.f;
        if (r < row0 + rows) {
          if (A.bf16) load8<WD_BF16>(src_q + 32 * j, A.q_vec, v[j]);
          else load8<WD_FP16>(src_q + 32 * j, A.q_vec, v[j]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[j][e]));
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // the largest component of a row lies in [2^14, 2^15)
      const int ex = min(max((int)(__float_as_uint(top) >> 23) - 127, -100), 113);
      const float up = __uint_as_float((uint32_t)(14 - ex + 127) << 23);
#pragma unroll
      for (int k = 0; k < NG; ++k) part[k] = 0.f;
#pragma unroll
      for (int j = 0; j < KW; ++j) {
#pragma unroll
        for (int e = 0; e < 8; ++e) { v[j][e] *= up; part[32 * j / G] += v[j][e]; }
        qf[x][j][0] = halves(v[j][0], v[j][4]);
        qf[x][j][1] = halves(v[j][1] * 0.0625f, v[j][5] * 0.0625f);
        qf[x][j][2] = halves(v[j][2], v[j][6]);
        qf[x][j][3] = halves(v[j][3] * 0.0625f, v[j][7] * 0.0625f);
      }
      const float c = fminf(fmaxf(A.scale_log2 * 4194304.f / up, 1e-37f), 1e38f);  // (a masked score times it stays -inf)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int rr = row0 + 8 * x + 2 * t + e;
        cn[x][e] = __shfl_sync(0xffffffffu, c, 8 * t + 4 * e);
        at[x][e] = rr < row0 + rows ? sq.len - A.q_len + rr / A.group : -1;
        M[x][e] = -1e30f;
        l[x][e] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < NG; ++k) {
        const float p = quad_sum(part[k]) * 2.384185791015625e-7f;  // 2^-22
#pragma unroll
        for (int e = 0; e < 2; ++e) { qs[x][k][e] = __shfl_sync(0xffffffffu, p, 8 * t + 4 * e); zs[x][k][e] = 0.f; }
#pragma unroll
        for (int e = 0; e < 4; ++e) cs[x][k][e] = 0.f;
      }
#pragma unroll
      for (int ws = 0; ws < NW; ++ws)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[x][ws][e / 8][e / 4 % 2][e % 4] = 0.f;
    }
    const int seen_by_all = sq.len - A.q_len + row0 / A.group, last_row = sq.len - A.q_len + (row0 + rows - 1) / A.group;
    const int hidden_from_some = max(last_row, -1) - A.window;  // (at least -2^31: a window is at most 2^31 - 1)

    int stage = 0;
#pragma unroll 1
    for (int j = 0; j < n; ++j) {
      // (copies run ahead by less than 32 tiles: the tile's bit is in this or the previous word)
      const int ahead = min(n - 1, j + ST - 1);
      const bool ok = ((ahead >> 5) == (j >> 5) ? good : good_before) >> (j & 31) & 1;
      if (ok && !dead) {
        const uint32_t parity = phase >> stage & 1;
        bool here = mb_try(bar + 8 * stage, parity);
        if (!__all_sync(0xffffffffu, here)) {
          const long long began = clock64();
          do {
            if (!here) here = mb_try(bar + 8 * stage, parity);
            dead = __any_sync(0xffffffffu, !here && clock64() - began > K4_SPIN_CLOCKS);
          } while (!dead && !__all_sync(0xffffffffu, here));
          if (dead) { set_status(A.p.status, ST_TIMEOUT); break; }
        }
        phase ^= 1u << stage;
        flying &= ~(1u << stage);
        const uint8_t* tile = ring + stage * S::TILE;
        const int pos0 = (tile0 + j * w) * 16;
        const bool edge = pos0 + 15 > seen_by_all || pos0 <= hidden_from_some;

        // scores: rows are tokens tok0 and tok0 + 8, columns rows of queries
        float x[NT][4];
        {
          uint32_t ka[KW], kb[KW], ma[NG], mb[NG];
          constexpr int n4 = D == 64 ? 2 : 4;
#pragma unroll
          for (int half = 0; half < KW / n4; ++half) {
            const int off = ((D == 256 ? half ^ (tok0 & 1) : 0) * 4 + t) * n4 * 4;
            uint32_t a[n4], c[n4];
            lds_words<n4>(tile + tok0 * (D / 2) + off, a);
            lds_words<n4>(tile + (tok0 + 8) * (D / 2) + off, c);
#pragma unroll
            for (int i = 0; i < n4; ++i) { ka[half * n4 + i] = a[i]; kb[half * n4 + i] = c[i]; }
          }
          lds_words<NG>(tile + 16 * D + tok0 * 4 * NG, ma);
          lds_words<NG>(tile + 16 * D + (tok0 + 8) * 4 * NG, mb);
#pragma unroll
          for (int k = 0; k < NG; ++k) {
            float acc[NT][4];
#pragma unroll
            for (int y = 0; y < NT; ++y)
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[y][e] = 0.f;
#pragma unroll
            for (int i = k * G / 32; i < (k + 1) * G / 32; ++i) {
#pragma unroll
              for (int s = 0; s < 2; ++s) {
                const uint32_t a = s ? ka[i] >> 6 : ka[i] << 2, c = s ? kb[i] >> 6 : kb[i] << 2;
#pragma unroll
                for (int y = 0; y < NT; ++y)
                  mma_f16(acc[y], a & 0x003c003cu, c & 0x003c003cu, a & 0x03c003c0u, c & 0x03c003c0u, qf[y][i][2 * s], qf[y][i][2 * s + 1]);
              }
            }
            const float2 sa = meta_values(ma[k], A.bf16), sc = meta_values(mb[k], A.bf16);
#pragma unroll
            for (int y = 0; y < NT; ++y)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float2 m = e < 2 ? sa : sc;
                const float z = k ? fmaf(m.y, qs[y][k][e & 1], x[y][e]) : m.y * qs[y][k][e & 1];
                x[y][e] = fmaf(m.x, acc[y][e], z);
              }
          }
        }
        // scales and zeros of the values of the same two tokens
        float2 va[NG], vb[NG];
        {
          uint32_t ma[NG], mb[NG];
          lds_words<NG>(tile + 16 * D + 64 * NG + tok0 * 4 * NG, ma);
          lds_words<NG>(tile + 16 * D + 64 * NG + (tok0 + 8) * 4 * NG, mb);
#pragma unroll
          for (int k = 0; k < NG; ++k) { va[k] = meta_values(ma[k], A.bf16); vb[k] = meta_values(mb[k], A.bf16); }
        }
        if (edge) {
          const int p0 = pos0 + tok0, p1 = p0 + 8;
          // Tokens that nobody sees may hold anything, and one that some rows see may hold NaN: neither must meet a weight of zero.
          bool any0 = false, any1 = false;
          const float nan = __int_as_float(0x7fffffff);
#pragma unroll
          for (int y = 0; y < NT; ++y)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int hi = at[y][e], lo = max(hi, -1) - A.window;
              const bool on0 = p0 <= hi && p0 > lo, on1 = p1 <= hi && p1 > lo;
              if (!on0) x[y][e] = -INFINITY;
              if (!on1) x[y][e + 2] = -INFINITY;
              any0 |= on0; any1 |= on1;
#pragma unroll
              for (int k = 0; k < NG; ++k)
                if ((on0 && !(fabsf(va[k].x) + fabsf(va[k].y) < INFINITY)) || (on1 && !(fabsf(vb[k].x) + fabsf(vb[k].y) < INFINITY))) zs[y][k][e] = nan;
            }
          any0 |= __shfl_xor_sync(0xffffffffu, any0, 1); any1 |= __shfl_xor_sync(0xffffffffu, any1, 1);
          any0 |= __shfl_xor_sync(0xffffffffu, any0, 2); any1 |= __shfl_xor_sync(0xffffffffu, any1, 2);
#pragma unroll
          for (int k = 0; k < NG; ++k) {
            if (!any0 || !(fabsf(va[k].x) + fabsf(va[k].y) < INFINITY)) va[k] = make_float2(0.f, 0.f);
            if (!any1 || !(fabsf(vb[k].x) + fabsf(vb[k].y) < INFINITY)) vb[k] = make_float2(0.f, 0.f);
          }
        }
        // weights relative to M, which moves only when a weight times its scale leaves what fp16 holds
        float big0 = 8.67361737988403547e-19f, big1 = big0;  // 2^-60: weights themselves stay below 2^74
#pragma unroll
        for (int k = 0; k < NG; ++k) { big0 = fmaxf(big0, va[k].x); big1 = fmaxf(big1, vb[k].x); }
        float p[NT][4], most = 0.f;
#pragma unroll
        for (int y = 0; y < NT; ++y)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[y][e] = ex2(fmaf(x[y][e], cn[y][e & 1], -M[y][e & 1]));
            most = fmaxf(most, p[y][e] * (e < 2 ? big0 : big1));
          }
        if (__any_sync(0xffffffffu, most > 16384.f)) {
          const float lg0 = log2f(big0) - 4.f, lg1 = log2f(big1) - 4.f;
#pragma unroll
          for (int y = 0; y < NT; ++y)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float m = rows_max(fmaxf(fmaf(x[y][e], cn[y][e], lg0), fmaf(x[y][e + 2], cn[y][e], lg1)));
              const float to = fmaxf(M[y][e], m), f = ex2(M[y][e] - to);
              M[y][e] = to;
              l[y][e] *= f;
#pragma unroll
              for (int k = 0; k < NG; ++k) { zs[y][k][e] *= f; cs[y][k][e] *= f; cs[y][k][e + 2] *= f; }
#pragma unroll
              for (int i = 0; i < 4 * NW; ++i) { o[y][i / 4][i / 2 % 2][i % 2][e] *= f; o[y][i / 4][i / 2 % 2][i % 2][e + 2] *= f; }
              p[y][e] = ex2(fmaf(x[y][e], cn[y][e], -to));
              p[y][e + 2] = ex2(fmaf(x[y][e + 2], cn[y][e], -to));
            }
        }
        // Weights times scales, rounded to fp16 for the product with the codes.  The codes count from the middle of their range, 8: the
        // rounding then weighs s |u - 8|, about a value's own size.  8 sum(p s) is taken off with the rounded weights (a product with
        // ones), and added back, unrounded, with the zeros.
        uint32_t pf[NT][NG][2];
#pragma unroll
        for (int y = 0; y < NT; ++y) {
#pragma unroll
          for (int e = 0; e < 2; ++e) l[y][e] += p[y][e] + p[y][e + 2];
#pragma unroll
          for (int k = 0; k < NG; ++k) {
            const float z0 = fmaf(va[k].x, 8.f, va[k].y), z1 = fmaf(vb[k].x, 8.f, vb[k].y);
#pragma unroll
            for (int e = 0; e < 2; ++e) zs[y][k][e] = fmaf(p[y][e], z0, fmaf(p[y][e + 2], z1, zs[y][k][e]));
            pf[y][k][0] = transpose8(halves(p[y][0] * va[k].x, p[y][1] * va[k].x));
            pf[y][k][1] = transpose8(halves(p[y][2] * vb[k].x, p[y][3] * vb[k].x));
            mma_f16(cs[y][k], 0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u, pf[y][k][0], pf[y][k][1]);
          }
        }
        // values: rows are components, summed over the tokens t, 7 - t, 8 + t, 15 - t of the lane
        {
          const uint8_t* base = tile + 16 * (D / 2);
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
                const int k = (64 * ws + 32 * half) / G;
                const uint32_t a0 = (s ? a >> 2 : a << 6) & 0x03c003c0u, a1 = (s ? a >> 6 : a << 2) & 0x03c003c0u;
                const uint32_t c0 = (s ? c >> 2 : c << 6) & 0x03c003c0u, c1 = (s ? c >> 6 : c << 2) & 0x03c003c0u;
#pragma unroll
                for (int y = 0; y < NT; ++y)
                  mma_f16(o[y][ws][half][s], a0, a1, c0, c1, pf[y][k][0], pf[y][k][1]);
              }
            }
        }
      }
      __syncwarp();
      if (j + ST < n) copy(j + ST, stage);
      stage = stage + 1 == ST ? 0 : stage + 1;
    }

    // the warp's sums, in shared memory
#pragma unroll
    for (int y = 0; y < NT; ++y)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float sum_l = rows_sum(l[y][e]);
        float z[NG];
#pragma unroll
        for (int k = 0; k < NG; ++k) z[k] = fmaf(-8.f, cs[y][k][e], rows_sum(zs[y][k][e]));
        float* line = piece + (8 * y + 2 * t + e) * S::LINE;
#pragma unroll
        for (int ws = 0; ws < NW; ++ws)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const float zz = z[(64 * ws + 32 * half) / G];
            const auto& a = o[y][ws][half];
            *reinterpret_cast<float4*>(line + 64 * ws + 32 * half + 4 * g) =
                make_float4(fmaf(a[0][e], 262144.f, zz), fmaf(a[0][e + 2], 262144.f, zz), fmaf(a[1][e], 262144.f, zz), fmaf(a[1][e + 2], 262144.f, zz));
          }
        if (g == 0) { line[D] = M[y][e]; line[D + 1] = sum_l; }
      }
    if (lane == 0) s_dead[warp] = dead;  // (a copy that is still on its way may land on the piece)
    team_sync();
    // the team's sums: to the output, or as a piece to the workspace
    const bool whole = seg == sq.tiles;
    const long long u0 = first + (long long)unit * sq.tiles;
    const int i0 = (int)(u0 / share), i1 = (int)((u0 + sq.tiles - 1) / share);
    float* slot = A.part + (long long)(2 * team + (team == i0)) * (S::PIECE / 4);
    const float* group_pieces = reinterpret_cast<const float*>(smem + (warp - wi) * S::RING);
    for (int x = wi * 32 + lane; x < rows * (D / 4); x += 32 * w) {
      const int r = x / (D / 4), c = x % (D / 4) * 4;
      const float* line = group_pieces + r * S::LINE;
      float m = -INFINITY, sum_l = 0.f;
      for (int i = 0; i < w; ++i) m = fmaxf(m, line[i * (S::RING / 4) + D]);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int i = 0; i < w; ++i) {
        const float* from = line + i * (S::RING / 4);
        const float f = s_dead[warp - wi + i] ? __int_as_float(0x7fffffff) : ex2(from[D] - m);
        const float4 y = *reinterpret_cast<const float4*>(from + c);
        sum_l = fmaf(f, from[D + 1], sum_l);
        v = make_float4(fmaf(f, y.x, v.x), fmaf(f, y.y, v.y), fmaf(f, y.z, v.z), fmaf(f, y.w, v.w));
      }
      if (whole) k4_put(A, b, h, row0 + r, D, c, v, m, sum_l);
      else {
        float* to = slot + r * S::LINE;
        __stcg(reinterpret_cast<float4*>(to + c), v);
        if (c == 0) __stcg(reinterpret_cast<float2*>(to + D), make_float2(m, sum_l));
      }
    }
    if (!whole) {
      __threadfence();
      team_sync();
      int32_t* arrived = A.arrived + ((long long)b * per_seq + unit);
      if (wi == 0 && lane == 0) {
        const int have = atomicAdd(arrived, 1);
        s_last[warp] = have == i1 - i0;
        if (have == i1 - i0) *arrived = 0;
        __threadfence();
      }
      team_sync();
      if (s_last[warp - wi]) {
        __threadfence();
        for (int x = wi * 32 + lane; x < rows * (D / 4); x += 32 * w) {
          const int r = x / (D / 4), c = x % (D / 4) * 4;
          const float* line = A.part + r * S::LINE;
          float m = -INFINITY, sum_l = 0.f;
          for (int i = i0; i <= i1; ++i) m = fmaxf(m, __ldcg(line + (long long)(2 * i + (i == i0)) * (S::PIECE / 4) + D));
          float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
          for (int i = i0; i <= i1; ++i) {
            const float* from = line + (long long)(2 * i + (i == i0)) * (S::PIECE / 4);
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(from + D));
            const float4 y = __ldcg(reinterpret_cast<const float4*>(from + c));
            const float f = ex2(ml.x - m);
            sum_l = fmaf(f, ml.y, sum_l);
            v = make_float4(fmaf(f, y.x, v.x), fmaf(f, y.y, v.y), fmaf(f, y.z, v.z), fmaf(f, y.w, v.w));
          }
          k4_put(A, b, h, row0 + r, D, c, v, m, sum_l);
        }
      }
    }
    team_sync();
    fence_async_shared();  // (the next copies land where the piece was)
    pos += seg;
  }
  // a warp that gave up leaves no copy behind it
  if (dead) {
    for (int i = 0; i < ST; ++i) {
      if (!(flying >> i & 1)) continue;
      const long long began = clock64();
      while (!mb_try(bar + 8 * i, phase >> i & 1) && clock64() - began < K4_SPIN_CLOCKS) {}
    }
  }
}

}  // namespace ls
