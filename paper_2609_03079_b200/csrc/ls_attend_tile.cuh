// Attention over a paged cache on the 5th-generation tensor cores: tiles of 128 query rows by 128 keys.
//
// The rows of one key head fill a tile: (tokens, query heads of the group), 128 / group tokens at a time.  Work is cut into
// units, each a set of rows and a range of keys:
//   pair units    two row tiles of the whole batch against the shared prefix (rows of the batch exceed one tile),
//   single units  the one row tile of the whole batch against the shared prefix (they do not),
//   own units     the rows of one sequence against its own keys.
// All (unit, key tile) pairs stand in one line, in a fixed order; every CTA takes an equal share of the line by cost and may
// start and end inside a unit.  A piece (one unit on one worker) leaves its normalised output and its lse in a slot of the
// workspace; a second kernel joins the pieces of every row in a fixed order.  Nothing about the lengths is needed on the host.
//
// A CTA has two lanes, each with its own scores and outputs in tensor memory (2 x (128 + dim) columns), and works on both in
// turn: while the tensor cores multiply for one lane, the four warps of the other do its softmax.  In a pair the lanes share
// every key and value tile; elsewhere each lane has its own line of (unit, key tile).
//   warps 0-3, 4-7  softmax of lanes 0 and 1;
//   warps 8, 11     copy keys (and queries) and values to shared memory (tensor maps, a box per page, a ring of tiles each);
//   warps 9, 10     issue the products of lanes 0 and 1.
// Wide pieces (17 to 128 rows): S = Q K^T, one softmax thread per row, P over S in tensor memory, O += P V.
// Narrow pieces (up to 16 rows: one token of one sequence): S^T = K Q^T, one softmax thread per key, P^T through shared memory,
// O^T += V^T P^T; the few exponentials are spread over all threads, and products that are 16 wide instead of 128 take a quarter.
// A row's reference maximum follows its true maximum only when that has risen by more than 2^8: weights stay below 2^8, the
// final division makes the reference irrelevant, and the accumulator in tensor memory is almost never rescaled.  The weights are
// rounded to the 16-bit type because the product with the values takes them so (the values have no more bits); their sum is
// taken before the rounding.  In fp16, whose range is short, they are held 2^7 higher (at most 2^15): what is rounded to nothing, or
// to the steps of 2^-24 that fp16 ends in, lies 2^-32 and 2^-31 below the reference instead of 2^-25 and 2^-24.  (100000 keys at e^-17.5
// beside a strong one are a quarter of a percent, which would all be lost.)
//
// What bounds it (B200, measured rates 6462 GB/s and 1683 TFLOP/s): own units by memory as long as all CTAs work on them (one
// sequence of 100001 keys, 64 / 8 heads: 71 us, 5.7 TB/s, 0.89 of measured), by the latency of a piece's start and end (about six
// thousand cycles) where pieces are a few tiles long; pairs by the chain softmax -> P V -> Q K^T of a lane (3.6 thousand cycles
// for two 128 x 128 tiles against 2.05 of products: tensor memory has no room for a second set of scores; 4.2 before the values
// of half a tile were multiplied under the other half's weights).  64 sequences on a 65536-key prefix: 191 to 204 us,
// depending on the card, 680 to 725 TFLOP/s, 0.41 to 0.43 of measured.  A fifth of the warps' time was once spent waiting for instructions:
// the six programs are kept short (loops rolled, one copy of each), which was worth 10 to 20 %.
// Measured against the alternatives: narrow pieces by the wide program 71 -> 85 us (one long sequence) and 110 -> 127 (128
// sequences); keys and values copied by one warp 82 -> 91 us with pages of 16; own units in the order sequence by sequence
// instead of head by head 104 -> 116 (40 key heads); ls_attend_rows_kernel instead of all this 71 -> 1027, 110 -> 9773.
#pragma once
#include "ls_attend.cuh"
#include "ls_tmem.cuh"

namespace ls {

constexpr int AT_THREADS = 384;
constexpr int AT_KEYS = 128;
constexpr int AT_MAX_CTAS = 256;
constexpr long long AT_SPIN_CLOCKS = 4000LL * 1000 * 1000;  // about two seconds
// What a key tile costs a CTA, whose lanes take two at once, start and end of short pieces included, for a pair and for a lane.
// 3 : 2 against 4 : 2, in turn on one card: 64 sequences on a 65536-key prefix 197.5 us against 204, 128 on 8192 keys 109 against 111.
// With a window more, because rows then see parts of a tile, whose masks cost a pair twice the time: 16 sequences of 4 drafts whose
// windows start inside the prefix 48 us with 5 against 62 with 3.  Where the window leaves most of the prefix whole, 5 is too much:
// 128 sequences on 8192 keys with a window of 4096 88 us against 71, 64 of 4 tokens with 6000 133 against 124.
constexpr int AT_COST_PAIR = 3, AT_COST_PAIR_WINDOW = 5, AT_COST_LANE = 2;
constexpr int AT_SHARE = 4, AT_SHARE_WINDOW = 5;  // a CTA's least share: a pair's tile, and a tile for both lanes

// The bits [lo, hi) of a word, as far as they lie in it.
__device__ __forceinline__ uint32_t range_bits(int lo, int hi) {
  const int a = min(max(lo, 0), 32), b = min(max(hi, 0), 32);
  const uint32_t below_b = b == 32 ? ~0u : (1u << b) - 1, below_a = a == 32 ? ~0u : (1u << a) - 1;
  return below_b & ~below_a;
}

template <int D>
struct TileShape {
  static constexpr int KST = D == 128 ? 2 : 4, VST = D == 128 ? 3 : 4, STAGES = KST + VST;  // places for keys and for values
  static constexpr int TILE = AT_KEYS * D * 2;   // bytes of a key, value or query tile
  static constexpr int HALF = AT_KEYS * 128;     // bytes of 64 of its columns
  // weights of a narrow piece: [2 x 64 keys][32 rows] of 128 bytes, in the last rows of the lane's query buffer
  static constexpr int NARROW_SLOTS = D == 128 ? 3 : 2, P_AT = NARROW_SLOTS * 32 * 128, P_HALF = D == 128 ? HALF : 32 * 128;
  static constexpr int CTL = (2 + STAGES) * TILE;  // offset of the control block
  static constexpr int SMEM = CTL + 3 * 1024;
};

struct TileArgs {
  AttendArgs a;
  int32_t tq, tb;    // tokens of a row tile of the whole batch; tokens a copy of it brings (fewer if the batch is smaller)
  int32_t ts, rt;    // tokens of a row tile of one sequence, row tiles of a sequence
  int32_t pairs;     // pairs of row tiles of the whole batch, 0: single
  int32_t box;       // keys per copy: the largest power of two that divides the page, at most 128
  float *pre_o, *pre_lse;  // slots of pair units ([2][128] rows) or single units ([128] rows)
  float *own_o, *own_lse;  // slots of own units ([ts * group] rows)
  int32_t *pre_first, *pre_last, *own_first, *own_last;  // per unit: the worker of its first and last piece
  int32_t* plan;     // [1] key tiles of the prefix
  int32_t workers;   // two per CTA
  uint8_t* gave_up;  // [AT_MAX_CTAS], 8-byte aligned, per CTA: a wait of its gave up in this call
};

// a / b for a >= 0, b > 0 and a quotient below 2^22 (then the estimate is off by one at most): numbers of units, heads, rows and
// sequences, which the workspace bounds well below that.
__device__ __forceinline__ int quotient(int a, int b) {
  int q = (int)((float)a * __frcp_rn((float)b));
  const int r = a - q * b;
  return r < 0 ? q - 1 : r >= b ? q + 1 : q;
}

// The same for any quotient: a second estimate from what the first one leaves.
__device__ __forceinline__ int quotient31(int a, int b) {
  const int q = (int)((float)a * __frcp_rn((float)b)), r = a - q * b;  // (off by 2^-22 of itself: r fits)
  return r >= 0 ? q + quotient(r, b) : q - quotient(b - 1 - r, b);
}

// First key that any token of a sequence sees.  (The positions are cut at 0 before the window is taken off: a window may be as large as
// 32 bits allow, and a sequence shorter than q_len.)
__device__ __forceinline__ int first_seen(const AttendArgs& A, int len) {
  return A.window > 0 ? max(max(len - A.q_len + 1, 0) - A.window, 0) : 0;
}

// The keys of sequence b that are its own: [lo, hi) is what any of its tokens sees, tiles start at `origin`.
struct OwnKeys { int lo, hi, origin, tiles; };
__device__ __forceinline__ OwnKeys own_keys(const TileArgs& T, int len) {
  OwnKeys k;
  k.lo = max(first_seen(T.a, len), T.a.prefix);
  k.hi = len;
  k.origin = k.lo & -T.box;
  k.tiles = k.hi > k.lo ? (k.hi - k.origin + AT_KEYS - 1) / AT_KEYS : 0;
  return k;
}

// What every CTA derives from the lengths: its share of the line of work.  (The host has made sure that positions in the line
// fit 31 bits.)
struct Share {
  int pre_lo, pre_origin, pre_tiles;  // prefix keys that any token sees: [pre_lo, prefix)
  int pair0, pair1;                   // this CTA's (pair unit, tile) range
  int lane0[2], lane1[2];             // its lanes' ranges in the line of single and own units
  int own_h[2], own_b[2], own_r[2], own_t[2];  // where a lane's range starts, if among the own units: head, sequence, row tile, tile
  OwnKeys own_k[2];                   // ... and that sequence's keys
  int batch_pieces[2];                // pieces of each lane that are not of own units (they come first)
  int sparse;                         // at most a tile for each CTA: lane 1 alone works, and workers are numbered by CTA
};

// A piece: consecutive tiles of one unit on one lane.  The copying warp walks the line and leaves each piece here, with its
// queries, for the warps that multiply and the ones that do the softmax.
enum { AT_PAIR = 0, AT_SINGLE = 1, AT_OWN = 2 };
struct Piece {
  int kind, h, tok, ntok;    // key head, first token and number of tokens of the row tile
  int k0, tiles, lo, hi;     // first key, number of tiles; keys outside [lo, hi) are nobody's
  int unit, ends;            // number of the unit among its kind; bit 0: holds its first tile, bit 1: its last
  int narrow;                // at most AT_NARROW rows
};

constexpr int AT_NARROW = 16;

// Exponents: how far a score may lie above its row's reference, and by how much weights are held higher than 2^(score - reference).
constexpr float AT_RISE = 8.f;
template <int WD> constexpr float AT_LIFT = WD == WD_FP16 ? 7.f : 0.f;

// Walks one lane's line piece by piece.
struct Walk {
  int w, end;             // position in the current part of the line
  bool pairs;             // still in the part of the pairs
  int h, b, r;            // next own unit (b = -1: still among the single ones): key head, sequence, row tile
  int tile, tiles;        // its next tile, its tiles (-1: to be looked up)
  int lo, hi, origin;     // keys of the current sequence or of the prefix
};

__device__ __forceinline__ void walk_start(const Share& S, Walk& W) {
  W.pairs = true;
  W.w = S.pair0;
  W.end = S.pair1;
}

// Takes the next piece of lane `lane`'s line; false at its end.
__device__ __forceinline__ bool walk_next(const TileArgs& T, const Share& S, int lane, Walk& W, Piece& P) {
  const AttendArgs& A = T.a;
  if (W.pairs && W.w == W.end) {
    W.pairs = false;
    W.w = S.lane0[lane]; W.end = S.lane1[lane];
    W.h = S.own_h[lane]; W.b = S.own_b[lane]; W.r = S.own_r[lane]; W.tile = S.own_t[lane];
    const OwnKeys k = S.own_k[lane];
    W.tiles = W.b < 0 ? -1 : k.tiles; W.lo = k.lo; W.hi = k.hi; W.origin = k.origin;
  }
  if (W.w >= W.end) return false;
  if (W.pairs || W.b < 0) {
    P.unit = quotient(W.w, S.pre_tiles);
    const int tile = W.w - P.unit * S.pre_tiles;
    P.tiles = min(S.pre_tiles - tile, W.end - W.w);
    P.ends = (tile == 0 ? 1 : 0) | (tile + P.tiles == S.pre_tiles ? 2 : 0);
    P.k0 = S.pre_origin + tile * AT_KEYS;
    P.lo = S.pre_lo; P.hi = A.prefix;
    if (W.pairs) {
      P.kind = AT_PAIR;
      P.narrow = 0;
      P.h = quotient(P.unit, T.pairs);
      P.tok = ((P.unit - P.h * T.pairs) * 2 + lane) * T.tq;
    } else {
      P.kind = AT_SINGLE;
      P.narrow = A.n_seqs * A.q_len * A.group <= AT_NARROW;
      P.h = P.unit;
      P.tok = 0;
      if ((P.ends & 2) && P.unit == A.kv_heads - 1) { W.h = 0; W.b = 0; W.r = 0; W.tile = 0; }
    }
    P.ntok = min(T.tq, A.n_seqs * A.q_len - P.tok);
  } else {
    if (W.tiles < 0) {
      for (;;) {  // (sequences without keys of their own have no units; the line ends before the last head's sequences do)
        const OwnKeys k = own_keys(T, attend_len(A, W.b, false));
        W.tiles = k.tiles; W.lo = k.lo; W.hi = k.hi; W.origin = k.origin;
        if (k.tiles > 0) break;
        if (++W.b == A.n_seqs) { W.b = 0; ++W.h; }
      }
    }
    P.kind = AT_OWN;
    P.narrow = T.ts * A.group <= AT_NARROW;
    P.tiles = min(W.tiles - W.tile, W.end - W.w);
    P.unit = (W.h * A.n_seqs + W.b) * T.rt + W.r;
    P.h = W.h;
    P.tok = W.b * A.q_len + W.r * T.ts;
    P.ntok = min(T.ts, A.q_len - W.r * T.ts);
    P.ends = (W.tile == 0 ? 1 : 0) | (W.tile + P.tiles == W.tiles ? 2 : 0);
    P.k0 = W.origin + W.tile * AT_KEYS;
    P.lo = W.lo; P.hi = W.hi;
    W.tile = 0;
    if ((P.ends & 2) && ++W.r == T.rt) {
      W.r = 0;
      W.tiles = -1;
      if (++W.b == A.n_seqs) { W.b = 0; ++W.h; }
    }
  }
  W.w += P.tiles;
  return true;
}

// Every thread of the CTA: the share of CTA c of n.
__device__ __forceinline__ void make_share(const TileArgs& T, Share& S, int* s_scan, int c, int n) {
  const AttendArgs& A = T.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nw = AT_THREADS / 32;
  const int per = (A.n_seqs + AT_THREADS - 1) / AT_THREADS;
  const int b0 = min(tid * per, A.n_seqs), b1 = min(b0 + per, A.n_seqs);
  int sum = 0, lo = A.prefix;  // own tiles (of one head and row tile) of this thread's sequences; first prefix key that they see
#pragma unroll 1
  for (int b = b0; b < b1; ++b) {
    const int len = attend_len(A, b, c == 0);
    sum += own_keys(T, len).tiles;
    if (len > 0) lo = min(lo, first_seen(A, len));
  }
  int incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  if (lane == 31) { s_scan[warp] = incl; s_scan[nw + warp] = lo; }
  __syncthreads();
  const int v = lane < nw ? s_scan[lane] : 0, vl = lane < nw ? s_scan[nw + lane] : A.prefix;
  const int before = incl - sum + __reduce_add_sync(0xffffffffu, lane < warp ? v : 0), total = __reduce_add_sync(0xffffffffu, v);
  lo = __reduce_min_sync(0xffffffffu, vl);
  const int origin = lo & -T.box;
  const int pre_tiles = A.prefix > lo ? (A.prefix - origin + AT_KEYS - 1) / AT_KEYS : 0;
  const int n_pair = A.kv_heads * T.pairs * pre_tiles, n_single = T.pairs ? 0 : A.kv_heads * pre_tiles;
  const int mult = A.kv_heads * T.rt, n_lane = n_single + total * mult;
  const bool windowed = A.window > 0;
  const int of_pair = windowed ? AT_COST_PAIR_WINDOW : AT_COST_PAIR, cost = n_pair * of_pair + n_lane * AT_COST_LANE;
  static_assert(AT_SHARE >= AT_COST_PAIR && AT_SHARE_WINDOW >= AT_COST_PAIR_WINDOW && AT_SHARE >= 2 * AT_COST_LANE, "least share");
  // Pieces of a unit have to be on consecutive workers: no worker between the first and the last may be empty.  Little work goes
  // to one lane of as many CTAs as there are tiles, what is a little more to fewer CTAs, each with a tile for both lanes.
  const bool sparse = n_pair == 0 && n_lane <= n;
  const int used = max(1, sparse ? n_lane : min(n, windowed ? cost / AT_SHARE_WINDOW : cost / AT_SHARE));
  const int base = quotient31(cost, used), rest = cost - base * used;  // CTA c takes the costs from c * base + c * rest / used on
  auto start = [&](int i) { i = min(i, used); return i * base + quotient(i * rest, used); };
  const int x0 = start(c), x1 = start(c + 1);
  auto pair_at = [&](int x) { return min(n_pair, windowed ? (x + of_pair - 1) / AT_COST_PAIR_WINDOW : (x + of_pair - 1) / AT_COST_PAIR); };
  auto lane_at = [&](int x) {
    x -= n_pair * of_pair;
    return x <= 0 ? 0 : min(n_lane, (x + AT_COST_LANE - 1) / AT_COST_LANE);
  };
  const int g0 = lane_at(x0), g1 = lane_at(x1), mid = g0 + (g1 - g0) / 2;
  if (tid == 0) {
    S.pre_lo = lo; S.pre_origin = origin; S.pre_tiles = pre_tiles; S.sparse = sparse;
    S.pair0 = pair_at(x0); S.pair1 = pair_at(x1);
    const int pp = pre_tiles > 0 && S.pair1 > S.pair0 ? quotient(S.pair1 - 1, pre_tiles) - quotient(S.pair0, pre_tiles) + 1 : 0;
    for (int l = 0; l < 2; ++l) {
      const int from = l ? mid : g0, to = min(l ? g1 : mid, n_single);
      S.lane0[l] = from; S.lane1[l] = l ? g1 : mid;
      if (from < n_single) S.own_b[l] = -1;
      S.batch_pieces[l] = pp + (to > from ? quotient(to - 1, pre_tiles) - quotient(from, pre_tiles) + 1 : 0);
    }
  }
  // Own units stand head by head, so that workers at the same place of their heads read neighbouring rows of the same tokens.
  const int line = total * T.rt;  // of one head
  for (int l = 0; l < 2; ++l) {   // the thread whose sequences hold the start of a lane's range finds it
    const int w = (l ? mid : g0) - n_single;
    if (w < 0 || line == 0) continue;
    const int h = quotient(w, line), at = w - h * line;
    int acc = before * T.rt;
    if (at < acc || at >= acc + sum * T.rt) continue;
#pragma unroll 1
    for (int b = b0; b < b1; ++b) {
      const OwnKeys k = own_keys(T, attend_len(A, b, false));
      const int t = k.tiles;
      if (at < acc + t * T.rt) {
        S.own_h[l] = h;
        S.own_b[l] = b;
        S.own_k[l] = k;
        S.own_r[l] = quotient(at - acc, t);
        S.own_t[l] = (at - acc) - S.own_r[l] * t;
        break;
      }
      acc += t * T.rt;
    }
  }
}

// (Out of line, like everything that is not on the way of every tile: a CTA's warps run six different programs, and what does not
// stay in the instruction cache is fetched through a memory system that the copies keep saturated.)
__device__ __forceinline__ bool tile_wait(uint32_t bar, uint32_t parity, volatile int* dead, int* status) {
  const long long t0 = clock64();
  bool got;
  while (!(got = mb_try(bar, parity))) {
    if (*dead) break;
    if (clock64() - t0 > AT_SPIN_CLOCKS) { *dead = 1; set_status(status, ST_TIMEOUT); break; }
  }
  return __all_sync(0xffffffffu, got);
}

// What a copying warp knows of a lane.
struct Feed {
  Walk w;
  Piece p, next;     // the piece of the current tile, and the one behind it
  int left, batch;   // tiles behind the current one; key of the first box whose page number is at hand
  int more, fresh;   // `next` is one; the current tile is the first of its piece
  int turn, same, key;  // the next batch of page numbers becomes the current one; the one to fetch: of this piece?, its first key
};

// Control block of a CTA, behind the tiles in shared memory.
template <int NST>
struct TileCtl {
  unsigned long long full[2][NST], empty[NST], qfull[2][4], qempty[2][4], s[2][2], p[2], p_half[2], o[2], turn[2], done[2];
  Share share;
  int scan[2 * AT_THREADS / 32];
  Piece piece[2][4];
  // narrow pieces: maxima and sums of each warp's keys.  (Places of their own: a warp may be at the end of a piece, with its sums,
  // while another one still reads the maxima of the last tile; no barrier of the four stands between.)
  float top[2][4][AT_NARROW], sum[2][4][AT_NARROW];
  int lo[2][AT_NARROW], hi[2][AT_NARROW];  // ... keys of each row, relative to the piece's first
  Feed feed[2][2];            // of the warps that copy keys and values, for each lane
  uint32_t tmem;
  volatile int dead;
};

template <int WD, int D>
__global__ void __launch_bounds__(AT_THREADS, 1)
    ls_attend_tile_kernel(const __grid_constant__ TileArgs T, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                          const __grid_constant__ CUtensorMap map_q_all, const __grid_constant__ CUtensorMap map_q_own) {
  using TS = TileShape<D>;
  constexpr int NST = TS::STAGES;
  extern __shared__ __align__(1024) unsigned char dyn[];
  static_assert(sizeof(TileCtl<NST>) <= TS::SMEM - TS::CTL, "control block");
  TileCtl<NST>& C = *reinterpret_cast<TileCtl<NST>*>(dyn + TS::CTL);
  Share& S = C.share;
  const AttendArgs& A = T.a;
  const int tid = threadIdx.x, lane_id = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const uint32_t q_base = saddr(dyn), ring = q_base + 2 * TS::TILE;
  const uint32_t b_full = saddr(C.full), b_empty = saddr(C.empty), b_qfull = saddr(C.qfull), b_qempty = saddr(C.qempty), b_s = saddr(C.s),
                 b_p = saddr(C.p), b_ph = saddr(C.p_half), b_o = saddr(C.o), b_turn = saddr(C.turn), b_done = saddr(C.done);
  if (warp == 0) {
    if (lane_id < 2 * NST) mb_init(b_full + 8 * lane_id, 1);
    if (lane_id < NST) mb_init(b_empty + 8 * lane_id, 2);
    if (lane_id < 8) { mb_init(b_qfull + 8 * lane_id, 1); mb_init(b_qempty + 8 * lane_id, 5); }
    if (lane_id < 4) mb_init(b_s + 8 * lane_id, 1);
    if (lane_id < 2) { mb_init(b_p + 8 * lane_id, 4); mb_init(b_ph + 8 * lane_id, 4); mb_init(b_o + 8 * lane_id, 1); mb_init(b_turn + 8 * lane_id, 1); mb_init(b_done + 8 * lane_id, 1); }
    if (lane_id == 0) C.dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_shared();
  }
  if (warp == 8 && lane_id < 4) tma_prefetch_map(lane_id == 0 ? &map_k : lane_id == 1 ? &map_v : lane_id == 2 ? &map_q_all : &map_q_own);
  asm volatile("griddepcontrol.wait;" ::: "memory");  // (all before this overlaps the end of the kernel in front)
  if (q_base & 1023) {  // (swizzled tiles need it; the first byte of a block's shared memory has it)
    if (tid == 0) { set_status(A.status, ST_INTERNAL); T.gave_up[blockIdx.x] = 1; }
    return;
  }
  make_share(T, S, C.scan, blockIdx.x, gridDim.x);
  __syncthreads();
  // (the copying warps, which have no use for tensor memory, do not wait for it)
  uint32_t tmem = 0;
  if (warp != 8 && warp != 11) {
    if (warp == 9) tm_alloc(saddr(&C.tmem), 512);
    tm_fence_before();
    group_sync(3, AT_THREADS - 64);
    tm_fence_after();
    tmem = C.tmem;
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // Bounded wait of a whole warp: false (for all of it) once any wait of the CTA has given up.
  auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
    if (__all_sync(0xffffffffu, mb_try(bar, parity))) return true;
    return tile_wait(bar, parity, &C.dead, A.status);
  };

  // Tiles of the lanes; the first n_pair of both are pairs.
  const int n_pair = S.pair1 - S.pair0;
  const int cnt0 = n_pair + S.lane1[0] - S.lane0[0], cnt1 = n_pair + S.lane1[1] - S.lane0[1];
  // Query tiles: rows of the whole batch take a lane's whole buffer; a sequence's rows take a slot of it, so that the copies run
  // ahead by several pieces where these rows are few.  (A slot's product may read 128 rows: what lies behind is ignored.)
  // Piece i of a lane is in slot 0 if it is one of the first batch_pieces, else in slot (i - batch_pieces) % q_slots; the slot's
  // barriers count the copy, and its release by the last product and by the four softmax warps.  The weights of
  // narrow pieces are behind the slots.
  const int q_rows = T.ts * A.group, q_slots = q_rows <= 32 ? TS::NARROW_SLOTS : q_rows <= 64 ? 2 : 1, q_step = q_rows <= 32 ? 32 * 128 : 64 * 128;
  struct Slots {
    int batch, n;
    uint32_t slot, par;
    __device__ __forceinline__ Slots(int batch_pieces, int slots, uint32_t parity) : batch(batch_pieces), n(slots), slot(0), par(parity) {}
    __device__ __forceinline__ uint32_t parity() const { return (par >> slot) & 1; }
    __device__ __forceinline__ void next() {
      par ^= 1u << slot;
      if (batch > 0) { --batch; return; }  // (the first own piece is in slot 0 too)
      if (++slot == (uint32_t)n) slot = 0;
    }
  };
  bool ok = true;
  if (warp == 8 || warp == 11) {
    // ---- copies: warp 8 keys, in rounds of a tile for each lane (a pair's once), and the queries of each piece; warp 11 values.
    // (Lanes of a warp issue a copy each, but are served one after the other: with pages of 16 tokens a tile takes sixteen, which
    // one warp could not issue as fast as memory brings them.)
    // A lane's tiles have barriers of their own (a place of the ring is filled now for one lane, now for the other; a lane that
    // watched both kinds of fills could be two behind and take an old one for its own); a pair's are those of lane 0.
    // Page numbers come 32 boxes at a time, one to each thread, a batch ahead: the next batch of the piece, or the first of the
    // next piece (so the walk is a piece ahead).
    const bool keys = warp == 8;
    const CUtensorMap* map = keys ? &map_k : &map_v;
    const uint32_t places = keys ? TS::KST : TS::VST, base = keys ? 0 : TS::KST;
    Feed* const feeds = C.feed[keys ? 0 : 1];
    int pages0 = 0, pages1 = 0, next0 = 0, next1 = 0;  // page numbers of the two lanes: this batch, the next one
    uint32_t st = 0, st_par = 1;
    Slots Q0(S.batch_pieces[0], q_slots, 15), Q1(S.batch_pieces[1], q_slots, 15);
    const int nbox = AT_KEYS / T.box, box_shift = 31 - __clz(T.box);
    const int my_box = lane_id & (nbox - 1), my_half = lane_id / nbox;
    const bool page_pow2 = (A.page & (A.page - 1)) == 0;
    const int page_shift = 31 - __clz(A.page);
    auto page_index = [&](int key) { return page_pow2 ? key >> page_shift : key / A.page; };
    // (the prefix is read again by other rows, a sequence's own keys are not)
    const uint64_t l2_keep = l2_evict_last(), l2_once = l2_evict_first();
    auto fetch_pages = [&](const Piece& p, int key) {  // (no branch around the load: nothing waits for it here)
      key += lane_id * T.box;
      const bool on = key < p.hi && key + T.box > p.lo;
      const int32_t* tab = p.kind == AT_OWN ? A.table + (long long)(A.q_len == 1 ? p.tok : p.tok / A.q_len) * A.table_stride : A.prefix_pages;
      return *(on ? tab + page_index(key) : A.seq_len);
    };
    // Both lanes go on to their next tile, a thread for each ...
    auto advance = [&]() {
      __syncwarp();
      if (lane_id < 2) {
        Feed& F = feeds[lane_id];
        F.fresh = F.left == 0 && F.more;
        if (F.left > 0) {
          --F.left;
          F.p.k0 += AT_KEYS;
          F.turn = F.p.k0 >= F.batch + 32 * T.box;
        } else if (F.more) {
          F.p = F.next;
          F.left = F.p.tiles - 1;
          F.turn = 1;
        }
        if (F.turn) F.batch = F.p.k0;
      }
      __syncwarp();
      if (feeds[0].turn) pages0 = next0;
      if (feeds[1].turn) pages1 = next1;
    };
    // ... and, with that tile's copies under way, look ahead: for the piece behind a new one, and the next batch of page numbers.
    auto look = [&]() {
      __syncwarp();
      if (lane_id < 2) {
        Feed& F = feeds[lane_id];
        if (F.fresh) F.more = walk_next(T, S, lane_id, F.w, F.next);
        F.fresh = 0;
        F.key = F.batch + 32 * T.box;
        F.same = F.left > 0 && F.key < F.p.k0 + (F.left + 1) * AT_KEYS;
        if (!F.same) F.key = F.next.k0;
      }
      __syncwarp();
      if (feeds[0].turn) next0 = feeds[0].same || feeds[0].more ? fetch_pages(feeds[0].same ? feeds[0].p : feeds[0].next, feeds[0].key) : 0;
      if (feeds[1].turn) next1 = feeds[1].same || feeds[1].more ? fetch_pages(feeds[1].same ? feeds[1].p : feeds[1].next, feeds[1].key) : 0;
      __syncwarp();
      if (lane_id < 2) feeds[lane_id].turn = 0;
    };
    if (lane_id < 2) {
      Feed& F = feeds[lane_id];
      walk_start(S, F.w);
      F.p.k0 = F.next.k0 = F.left = F.batch = 0;
      F.more = F.fresh = F.turn = 1;
    }
#pragma unroll 1
    for (int x = -1; x < 2 * max(cnt0, cnt1); ++x) {
      const int l = x & 1, r = x >> 1;
      if (x >= 0 && l == 0) advance();
      if (x < 0 || r >= (l ? cnt1 : cnt0)) {
        if (l) look();
        continue;
      }
      const Feed& F = feeds[l];
      const bool own = F.p.kind == AT_OWN;
      if (keys && F.fresh) {
        const uint32_t slot = l ? Q1.slot : Q0.slot;
        ok = wait(b_qempty + 32 * l + 8 * slot, l ? Q1.parity() : Q0.parity());
        if (!ok) break;
        if (l) Q1.next();
        else Q0.next();
        if (lane_id == 0) {
          C.piece[l][slot] = F.p;
          const uint32_t full = b_qfull + 32 * l + 8 * slot;
          mb_expect(full, (own ? T.ts : T.tb) * A.group * D * 2);
#pragma unroll
          for (int f = 0; f < D / 64; ++f)
            tma_load3(q_base + l * TS::TILE + f * TS::HALF + slot * q_step, own ? &map_q_own : &map_q_all, f * 64, F.p.h * A.group, F.p.tok, full);
        }
        __syncwarp();
      }
      if (!(r < n_pair && l == 1)) {
        int page = __shfl_sync(0xffffffffu, l ? pages1 : pages0, ((F.p.k0 - F.batch) >> box_shift) + my_box);
        const int key = F.p.k0 + my_box * T.box;
        const bool on = my_half < D / 64 && key < F.p.hi && key + T.box > F.p.lo;
        const int count = __popc(__ballot_sync(0xffffffffu, on));
        if (on && (uint32_t)page >= (uint32_t)A.n_pages) { set_status(A.status, ST_BAD_INDEX); page = A.n_pages; }  // (reads as zeros)
        const uint32_t place = base + st, full = b_full + 8 * (place + (r >= n_pair ? NST * l : 0));
        ok = wait(b_empty + 8 * place, st_par);
        if (!ok) break;
        if (lane_id == 0) mb_expect(full, count * T.box * 128);
        __syncwarp();
        if (on)
          tma_load4(ring + place * TS::TILE + my_half * TS::HALF + my_box * T.box * 128, map, my_half * 64, key - page_index(key) * A.page, F.p.h, page, full,
                    own ? l2_once : l2_keep);
        if (++st == places) { st = 0; st_par ^= 1; }
      }
      if (l) look();
    }
  } else if (warp >= 9) {
    // ---- products of one lane, issued by one thread.  Wide tiles: O += P V of round r - 1, then S = Q K^T of round r, which
    // overwrites P; the lanes take strict turns on pairs, so that one lane's products run together while the other lane is in
    // its softmax (products of both lanes mixed would end at the same time, and the two softmaxes share the same cycles).
    // Narrow tiles: S^T = K Q^T of round r first (two buffers of scores), then O^T += V^T P^T of round r - 1.
    // The warp clears value rows that are nobody's (whatever the page holds there, its weight of zero must not meet an infinity;
    // in a pair both lanes clear, the same).  A tile's two arrivals on `empty` are the commits of the pair's two lanes, or the
    // commit of the one lane that reads it and an arrival of its own in place of the other.
    constexpr int TYPE = WD == WD_BF16;
    constexpr uint32_t ID_S = mma_idesc(TYPE, 128, AT_KEYS, false, false), ID_O = mma_idesc(TYPE, 128, D, false, true);
    constexpr uint32_t ID_ST = mma_idesc(TYPE, 128, AT_NARROW, false, false), ID_OT = mma_idesc(TYPE, 128, AT_NARROW, true, false);
    const int l = warp - 9;
    const int cnt = l ? cnt1 : cnt0;
    const uint32_t t_s = uniform32(tmem + l * AT_KEYS), t_o = uniform32(tmem + 256 + l * D);
    const uint64_t p_desc = uniform64(smem_desc(q_base + l * TS::TILE + TS::P_AT, 16));
    Slots Q(S.batch_pieces[l], q_slots, 0);
    int left = 0, k0 = 0, lo = 0, hi = 0;   // of the current piece: tiles to come, first key of the next; keys of anybody
    int narrow = 0, vk0 = 0, vlo = 0, vhi = 0, vnarrow = 0;  // v*: of the tile whose values are still to be multiplied
    bool vfresh = true;
    uint32_t q_slot = 0, kst = 0, vst = 0, par0 = 0, par1 = 0;  // par*: parity of each place's next fill, by set of barriers
    for (int r = 0; r <= cnt; ++r) {
      // places in the rings: lane 0's tile, then lane 1's, a pair's once
      const bool vpair = r <= n_pair, kpair = r < n_pair;
      const uint32_t kplace = kst + (l == 1 && !kpair && r < cnt0), vplace = vst + (l == 1 && !vpair && r <= cnt0);
      const uint32_t kslot = kplace >= TS::KST ? kplace - TS::KST : kplace, vslot = TS::KST + (vplace >= TS::VST ? vplace - TS::VST : vplace);
      auto filled = [&](uint32_t slot, bool pair) -> bool {
        const bool set0 = pair || l == 0;
        const uint32_t par = set0 ? par0 : par1;
        if (set0) par0 ^= 1u << slot;
        else par1 ^= 1u << slot;
        if (!wait(b_full + 8 * (set0 ? slot : NST + slot), (par >> slot) & 1)) return false;
        if (!pair && elect_one()) mb_arrive(b_empty + 8 * slot);
        return true;
      };
      bool kfresh = false;
      auto scores = [&]() -> bool {
        const uint32_t slot = kslot;
        kfresh = left == 0;
        if (kfresh) {
          q_slot = Q.slot;
          if (!wait(b_qfull + 32 * l + 8 * q_slot, Q.parity())) return false;
          Q.next();
          const Piece& P = C.piece[l][q_slot];
          left = P.tiles; k0 = P.k0; lo = P.lo; hi = P.hi; narrow = P.narrow;
        }
        if (!filled(slot, kpair)) return false;
        --left;
        tm_fence_after();
        const uint32_t q = q_base + l * TS::TILE + q_slot * q_step, k = ring + slot * TS::TILE;
        const uint64_t a = uniform64(smem_desc(narrow ? k : q, 16)), b = uniform64(smem_desc(narrow ? q : k, 16));
        const uint32_t id = uniform32(narrow ? ID_ST : ID_S), d = uniform32(narrow ? t_s + (r & 1) * 32 : t_s);
        if (elect_one()) {
#pragma unroll
          for (int c = 0; c < D / 16; ++c) {
            const uint32_t off = ((c / 4) * TS::HALF + (c % 4) * 32) >> 4;
            tm_mma_ss(d, a + off, b + off, id, c > 0);
          }
          tm_commit(b_s + 16 * l + 8 * (r & 1));
          tm_commit(b_empty + 8 * slot);
          if (left == 0) tm_commit(b_qempty + 32 * l + 8 * q_slot);
        }
        __syncwarp();
        return true;
      };
      auto outputs = [&]() -> bool {
        const uint32_t slot = vslot;
        if (!filled(slot, vpair)) return false;
        if (vk0 < vlo || vk0 + AT_KEYS > vhi) {
          for (int c = lane_id; c < AT_KEYS; c += 32) {
            if (vk0 + c >= vlo && vk0 + c < vhi) continue;
            for (int f = 0; f < D / 64; ++f)
              for (int j = 0; j < 8; ++j)
                asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(ring + slot * TS::TILE + f * TS::HALF + c * 128 + j * 16), "r"(0) : "memory");
          }
          fence_async_shared();
          __syncwarp();
        }
        if (!wait((vnarrow ? b_p : b_ph) + 8 * l, (r - 1) & 1)) return false;
        if (r <= n_pair && (l || r > 0) && !wait(b_turn + 8 * l, (l ? r : r - 1) & 1)) return false;
        tm_fence_after();
        const uint64_t v = uniform64(smem_desc(ring + slot * TS::TILE, TS::HALF));
        if (elect_one()) {
          if (vnarrow) {
            // (64 columns of values fill a 128-row product twice: both blocks of 64 are the same one)
            const uint64_t va = D == 128 ? v : v & ~((uint64_t)0x3fff << 16);
#pragma unroll
            for (int k = 0; k < AT_KEYS / 16; ++k)
              tm_mma_ss(t_o, va + k * (2048 >> 4), p_desc + (((k / 4) * TS::P_HALF + (k % 4) * 32) >> 4), ID_OT, !(vfresh && k == 0));
            tm_commit(b_o + 8 * l);
            tm_commit(b_empty + 8 * slot);
          } else {
#pragma unroll
            for (int k = 0; k < AT_KEYS / 32; ++k) tm_mma_ts(t_o, t_s + k * 8, v + k * (2048 >> 4), ID_O, !(vfresh && k == 0));
          }
        }
        if (!vnarrow) {
          __syncwarp();
          if (!wait(b_p + 8 * l, (r - 1) & 1)) return false;
          tm_fence_after();
          if (elect_one()) {
#pragma unroll
            for (int k = AT_KEYS / 32; k < AT_KEYS / 16; ++k) tm_mma_ts(t_o, t_s + k * 8, v + k * (2048 >> 4), ID_O, true);
            tm_commit(b_o + 8 * l);
            tm_commit(b_empty + 8 * slot);
          }
        }
        __syncwarp();
        return true;
      };
      // Scores first only if their operands are there (the outputs' weights come soon, keys may come late), and never behind a
      // wide tile, whose weights they would overwrite.
      bool scores_first = r > 0 && vnarrow && r < cnt;
      if (scores_first) {
        scores_first = mb_test(b_full + 8 * (l ? NST + kslot : kslot), ((l ? par1 : par0) >> kslot) & 1);
        if (left == 0) scores_first = scores_first && mb_test(b_qfull + 32 * l + 8 * Q.slot, Q.parity());
        scores_first = __all_sync(0xffffffffu, scores_first);
      }
      bool good = true;
      if (r == 0 && l == 1 && n_pair > 0) good = wait(b_turn + 8, 0);
#pragma unroll 1
      for (int x = 0; x < 2 && good; ++x) {
        if ((x == 0) == scores_first) { if (r < cnt) good = scores(); }
        else if (r > 0) good = outputs();
      }
      if (!good) break;
      vk0 = k0; vlo = lo; vhi = hi; vnarrow = narrow; vfresh = kfresh;
      k0 += AT_KEYS;
      if (r <= n_pair && elect_one()) mb_arrive(b_turn + 8 * (1 - l));
      kst += (r < cnt0) + (r < cnt1 && !kpair);
      if (kst >= TS::KST) kst -= TS::KST;
      if (r > 0) vst += (r <= cnt0) + (r <= cnt1 && !vpair);
      if (vst >= TS::VST) vst -= TS::VST;
    }
    // every arrival that the tensor cores owe this block has come when the last one has
    if (elect_one()) tm_commit(b_done + 8 * l);
    wait(b_done + 8 * l, 0);
  } else {
    // ---- softmax.  A wait that gives up does not change the way of a warp through a piece (its four warps meet at barriers);
    // they all leave before the next one.
    const int l = warp >> 2, quad = warp & 3, row = quad * 32 + lane_id;
    const int cnt = l ? cnt1 : cnt0;
    const uint32_t t_s = tmem + (quad << 21) + l * AT_KEYS, t_o = tmem + (quad << 21) + 256 + l * D;
    Slots Q(S.batch_pieces[l], q_slots, 0);
    const float scale = A.scale_log2;
    constexpr float LIFT = AT_LIFT<WD>;
    const int worker = S.sparse ? blockIdx.x : blockIdx.x * 2 + l;
    int n = 0;
    auto arrive_p = [&](uint32_t bar) {
      tm_fence_before();
      __syncwarp();
      if (lane_id == 0) mb_arrive(bar + 8 * l);
    };
    // Keys [lo, hi) that row x of a piece sees, relative to the piece's first.
    auto row_keys = [&](const Piece& P, int x, int& lo, int& hi) {
      const int t = P.tok + (P.ntok == 1 ? 0 : quotient(x, A.group)), b = A.q_len == 1 ? t : quotient(t, A.q_len);
      // (an own unit's last key is its sequence's last)
      hi = max((P.kind == AT_OWN ? P.hi : attend_len(A, b, false)) - A.q_len + (t - b * A.q_len) + 1, 0);
      lo = A.window > 0 ? max(hi - A.window, 0) : 0;
      if (P.kind == AT_OWN) lo = max(lo, A.prefix);
      else hi = min(hi, A.prefix);
      lo -= P.k0; hi -= P.k0;
    };
    // Where row 0 of a piece goes in the workspace; one thread notes which workers hold a unit.
    auto place_piece = [&](const Piece& P, float*& po, float*& pl) -> long long {
      if (P.kind == AT_OWN) {
        po = T.own_o; pl = T.own_lse;
        if (row == 0 && (P.ends & 1)) T.own_first[P.unit] = worker;
        if (row == 0 && (P.ends & 2)) T.own_last[P.unit] = worker;
        return (long long)(P.unit + worker) * (T.ts * A.group);
      }
      const bool pair = P.kind == AT_PAIR;
      const int wk = pair ? blockIdx.x : worker;
      po = T.pre_o; pl = T.pre_lse;
      const bool mark = row == 0 && !(pair && l == 1);
      if (mark && (P.ends & 1)) T.pre_first[P.unit] = wk;
      if (mark && (P.ends & 2)) T.pre_last[P.unit] = wk;
      return (pair ? (P.unit + wk) * 2LL + l : (long long)(P.unit + wk)) * 128;
    };

    // Narrow pieces: at most 16 rows.  The product is turned round, S^T = K Q^T: a thread has one key and the scores of all
    // rows, so that the few exponentials are spread over all 128 threads.  Weights go to shared memory as P^T's other operand.
    // The reference of a row is kept in what is added to the exponent, `off` = lift - reference; 3e38 stands for a row that has seen nothing, so that
    // its first score exceeds the reference too.  The rows' sums stay apart, by key, until the end of the piece.
    auto narrow_piece = [&](const Piece& P) {
      constexpr int NR = AT_NARROW;
      const int rows = P.ntok * A.group;
      const uint32_t p_base = q_base + l * TS::TILE + TS::P_AT + (quad >> 1) * TS::P_HALF;  // this thread's half of the keys
      const uint32_t p_chunk = (uint32_t)(row & 63) >> 3, p_byte = (row & 7) * 2;
      int my_lo = -0x7fffffff, my_hi = 0x7fffffff;
      if (lane_id < rows) { my_lo = C.lo[l][lane_id]; my_hi = C.hi[l][lane_id]; }
      int all_lo = __reduce_max_sync(0xffffffffu, my_lo), all_hi = __reduce_min_sync(0xffffffffu, my_hi);  // what every row sees
      float off[NR], sum[NR], my_off = 3e38f;  // my_off: of row `lane`
#pragma unroll
      for (int x = 0; x < NR; ++x) { off[x] = 3e38f; sum[x] = 0.f; }
      for (int j = 0; j < P.tiles; ++j, ++n, all_lo -= AT_KEYS, all_hi -= AT_KEYS) {
        wait(b_s + 16 * l + 8 * (n & 1), (n >> 1) & 1);
        if (n > 0) wait(b_o + 8 * l, (n - 1) & 1);  // (its weights are done with)
        tm_fence_after();
        uint32_t s[NR];
        tm_ld16(t_s + (n & 1) * 32, s);
        tm_wait_ld();
        tm_pin16(s);
        if (all_lo > 0 || all_hi < AT_KEYS) {
          const int key = j * AT_KEYS + row;
#pragma unroll
          for (int x = 0; x < NR; ++x)
            if (x < rows && (key < C.lo[l][x] || key >= C.hi[l][x])) s[x] = 0xff800000u;
        }
        bool rise = false;
#pragma unroll
        for (int x = 0; x < NR; ++x) rise |= x < rows && fmaf(__uint_as_float(s[x]), scale, off[x]) > AT_RISE + LIFT;
        if (group_any(1 + l, 128, rise)) {
          // the rows' true maxima: of each warp's keys, then of all (lane x of every warp keeps row x)
          float top = -INFINITY;
#pragma unroll
          for (int x = 0; x < NR; ++x) {
            const float v = warp_max(__uint_as_float(s[x]));
            if (lane_id == x) top = v;
          }
          if (lane_id < NR) C.top[l][quad][lane_id] = top;
          group_sync(1 + l, 128);
          if (lane_id < rows) {
            top = fmaxf(fmaxf(C.top[l][0][lane_id], C.top[l][1][lane_id]), fmaxf(C.top[l][2][lane_id], C.top[l][3][lane_id])) * scale;
            rise = top + my_off > AT_RISE + LIFT;
          } else rise = false;
          const float f = rise ? ex2(LIFT - top - my_off) : 1.f;
          if (rise) my_off = LIFT - top;
          uint32_t o[NR];
          if (j > 0) {
            tm_ld16(t_o, o);
            tm_wait_ld();
            tm_pin16(o);
          }
#pragma unroll
          for (int x = 0; x < NR; ++x) {
            const float fx = __shfl_sync(0xffffffffu, f, x);
            off[x] = __shfl_sync(0xffffffffu, my_off, x);
            sum[x] *= fx;
            o[x] = __float_as_uint(__uint_as_float(o[x]) * fx);
          }
          if (j > 0) {
            tm_st16(t_o, o);
            tm_wait_st();
          }
        }
        // (four rows at a time, whether there are as many or not: what a row that is not there leaves behind is not used)
#pragma unroll
        for (int g = 0; g < NR; g += 4)
          if (g < rows) {
            uint16_t w[4];
#pragma unroll
            for (int x = g; x < g + 4; ++x) {
              const float p = ex2(fmaf(__uint_as_float(s[x]), scale, off[x]));
              sum[x] += p;
              w[x - g] = narrow16<WD>(p);
            }
#pragma unroll
            for (int x = g; x < g + 4; ++x)
              asm volatile("st.shared.b16 [%0], %1;" ::"r"(p_base + x * 128 + ((p_chunk ^ (x & 7)) << 4) + p_byte), "h"(w[x - g]) : "memory");
          }
        fence_async_shared();
        arrive_p(b_p);
      }
      float my_sum = 0.f;
#pragma unroll
      for (int g = 0; g < NR; g += 4)
        if (g < rows) {
          float v[4];
#pragma unroll
          for (int x = 0; x < 4; ++x) v[x] = sum[g + x];
#pragma unroll
          for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int x = 0; x < 4; ++x) v[x] += __shfl_xor_sync(0xffffffffu, v[x], o);
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if (lane_id == g + x) C.sum[l][quad][g + x] = v[x];
        }
      uint32_t o[NR];
      wait(b_o + 8 * l, (n - 1) & 1);
      tm_fence_after();
      tm_ld16(t_o, o);
      group_sync(1 + l, 128);
      if (lane_id < rows) my_sum = (C.sum[l][0][lane_id] + C.sum[l][1][lane_id]) + (C.sum[l][2][lane_id] + C.sum[l][3][lane_id]);
      const float inv = my_sum == 0.f ? 0.f : 1.f / my_sum;
      float *po, *pl;
      const long long at = place_piece(P, po, pl);
      if (quad == 0 && lane_id < rows) pl[at + lane_id] = my_sum == 0.f ? -INFINITY : log2f(my_sum) - my_off;
      tm_wait_ld();
      tm_pin16(o);
#pragma unroll
      for (int g = 0; g < NR; g += 4)
        if (g < rows) {
#pragma unroll
          for (int x = g; x < g + 4; ++x) {
            const float f = __shfl_sync(0xffffffffu, inv, x);
            if (row < D && x < rows) po[(at + x) * D + row] = __uint_as_float(o[x]) * f;
          }
        }
      tm_fence_before();
    };

    while (n < cnt) {
      const uint32_t slot = Q.slot;
      bool good = wait(b_qfull + 32 * l + 8 * slot, Q.parity()) && !C.dead;
      Q.next();
      const Piece P = C.piece[l][slot];
      if (good && P.narrow && row < P.ntok * A.group) {
        int a, b;
        row_keys(P, row, a, b);
        C.lo[l][row] = a;
        C.hi[l][row] = b;
      }
      if (group_any(1 + l, 128, !good)) break;
      if (lane_id == 0) mb_arrive(b_qempty + 32 * l + 8 * slot);
      if (P.narrow) { narrow_piece(P); continue; }
      // Wide pieces: one thread per row.
      const bool live = row < P.ntok * A.group, warp_live = __any_sync(0xffffffffu, live);
      int lo = 0, hi = 0x7fffffff;  // keys this row sees, relative to the tile
      if (live) row_keys(P, row, lo, hi);
      float m = -INFINITY, sum = 0.f;
      for (int j = 0; j < P.tiles; ++j, ++n, lo -= AT_KEYS, hi -= AT_KEYS) {
        wait(b_s + 16 * l + 8 * (n & 1), (n >> 1) & 1);
        tm_fence_after();
        if (warp_live) {
          const bool masked = !__all_sync(0xffffffffu, lo <= 0 && hi >= AT_KEYS);
          const uint64_t scale2 = both(scale);
          uint64_t acc[2] = {0, 0};
          auto weights = [&](uint32_t* s, uint64_t off2) {  // 32 scores to 16 pairs of weights
#pragma unroll
            for (int c = 0; c < 32; c += 2) {
              const uint64_t x = fma2(pair32(s[c], s[c + 1]), scale2, off2);
              const float p0 = ex2(lo32(x)), p1 = ex2(hi32(x));
              acc[(c / 2) & 1] = add2(acc[(c / 2) & 1], pair32(__float_as_uint(p0), __float_as_uint(p1)));
              s[c / 2] = pack2<WD>(p0, p1);
            }
          };
          // Two passes over the scores: the maximum (all four quarters of the columns), then the weights.  The quarters 0 and 1 stay in
          // registers between the passes; 2 and 3 are read again (masked ones are written back first).  The weights of a
          // quarter go over scores that are in registers or done with.
          uint32_t s0[32], s1[32];
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
          for (int half = 1; half >= 0; --half) {
            tm_ld32(t_s + 64 * half, s0);
            tm_ld32(t_s + 64 * half + 32, s1);
            tm_wait_ld();
            tm_pin32(s0);
            tm_pin32(s1);
            if (masked) {
              const uint32_t on0 = range_bits(lo - 64 * half, hi - 64 * half), on1 = range_bits(lo - 64 * half - 32, hi - 64 * half - 32);
#pragma unroll
              for (int c = 0; c < 32; ++c) {
                if (!(on0 & 1u << c)) s0[c] = 0xff800000u;
                if (!(on1 & 1u << c)) s1[c] = 0xff800000u;
              }
              if (half) {
                tm_st32(t_s + 64, s0);
                tm_st32(t_s + 96, s1);
              }
            }
#pragma unroll
            for (int c = 0; c < 32; c += 2) {
              mx[(c / 2) & 1] = max3(mx[(c / 2) & 1], __uint_as_float(s0[c]), __uint_as_float(s0[c + 1]));
              mx[2 + ((c / 2) & 1)] = max3(mx[2 + ((c / 2) & 1)], __uint_as_float(s1[c]), __uint_as_float(s1[c + 1]));
            }
          }
          if (masked) tm_wait_st();
          const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
          const bool rise = live && top > m && (m == -INFINITY || (top - m) * scale > AT_RISE);
          if (__any_sync(0xffffffffu, rise)) {
            const float f = rise ? ex2((m - top) * scale) : 1.f;
            if (rise) { m = top; sum *= f; }
            if (j > 0) {
              wait(b_o + 8 * l, (n - 1) & 1);
              tm_fence_after();
#pragma unroll 1
              for (int c = 0; c < D / 32; ++c) {
                uint32_t o[32];
                tm_ld32(t_o + 32 * c, o);
                tm_wait_ld();
                tm_pin32(o);
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                tm_st32(t_o + 32 * c, o);
              }
            }
          }
          const float off = m == -INFINITY ? 0.f : fmaf(-m, scale, LIFT);
          const uint64_t off2 = both(off);
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {
            weights(s0, off2);
            tm_st16(t_s + 32 * half, s0);
            if (half == 0) tm_ld32(t_s + 64, s0);
            weights(s1, off2);
            tm_st16(t_s + 32 * half + 16, s1);
            if (half == 1) break;
            tm_ld32(t_s + 96, s1);
            tm_wait_st();  // the weights of the first 64 keys can be multiplied while the others are made
            arrive_p(b_ph);
            tm_wait_ld();
            tm_pin32(s0);
            tm_pin32(s1);
          }
          const uint64_t acc_all = add2(acc[0], acc[1]);
          sum += lo32(acc_all) + hi32(acc_all);
          tm_wait_st();
        } else arrive_p(b_ph);
        arrive_p(b_p);
      }
      // the piece is done: its output and lse go to the workspace
      wait(b_o + 8 * l, (n - 1) & 1);
      tm_fence_after();
      float *po, *pl;
      const long long at = place_piece(P, po, pl) + row;
      if (warp_live) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        if (live) pl[at] = sum == 0.f ? -INFINITY : fmaf(m, scale, log2f(sum) - LIFT);
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
          uint32_t o[32];
          tm_ld32(t_o + 32 * c, o);
          tm_wait_ld();
          tm_pin32(o);
          if (live) {
            float4* dst = reinterpret_cast<float4*>(po + at * D + 32 * c);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              dst[e] = make_float4(__uint_as_float(o[4 * e]) * inv, __uint_as_float(o[4 * e + 1]) * inv, __uint_as_float(o[4 * e + 2]) * inv,
                                   __uint_as_float(o[4 * e + 3]) * inv);
          }
        }
        tm_fence_before();
      }
    }
  }
  if (blockIdx.x == 0 && tid == 0) *T.plan = S.pre_tiles;
  __syncthreads();
  if (tid == 0) T.gave_up[blockIdx.x] = C.dead != 0;
  if (C.dead) {  // copies and products that are still in flight get time to land before the CTA's memory goes
    const long long t0 = clock64();
    while (clock64() - t0 < AT_SPIN_CLOCKS / 1000) {}
    __syncthreads();
  }
  tm_fence_after();
  if (warp == 9) tm_free(tmem, 512);
}

// ---- joins the pieces of every row in their order: WARPS warps per row take turns at its pieces ------------------------------
// (one warp where rows are many and have a few pieces each; eight where rows are few and may be cut into a hundred: 64 rows of 40
// pieces 85 -> 73 us for the whole call, 8192 rows of 5 pieces with eight 110 -> 131)
// Bound by latency: five dependent reads of L2, the first outputs asked for together with the weights.
template <int WD, int D, int WARPS>
__global__ void __launch_bounds__(256) ls_attend_tile_join_kernel(const TileArgs T) {
  const AttendArgs& A = T.a;
  const long long rows = (long long)A.n_seqs * A.q_len * A.heads;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = warp % WARPS;
  const long long row = (long long)blockIdx.x * (8 / WARPS) + warp / WARPS;
  __shared__ float s_acc[WARPS > 1 ? 8 : 1][D + 1];
  if (row >= rows) return;  // (a block of its own row when WARPS is 8: all of it returns)
  const int t = (int)(row / A.heads), hd = (int)(row - (long long)t * A.heads), h = hd / A.group, g = hd - h * A.group;
  const int b = t / A.q_len, i = t - b * A.q_len;
  long long pre_unit, pre_row, pre_step;
  if (T.pairs) {
    const int tile = t / T.tq;
    pre_unit = (long long)h * T.pairs + tile / 2;
    pre_row = (tile & 1) * 128 + (t - tile * T.tq) * A.group + g;
    pre_step = 256;
  } else {
    pre_unit = h;
    pre_row = t * A.group + g;
    pre_step = 128;
  }
  const int rt = i / T.ts;
  const long long own_unit = ((long long)h * A.n_seqs + b) * T.rt + rt, own_step = (long long)T.ts * A.group;
  const long long own_row = (i - rt * T.ts) * A.group + g;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // (with many rows the next kernel's blocks, waiting here early, were measured to cost more than their start takes)
  if (WARPS > 1) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  int n_pre = 0, n_own = 0;
  long long pre_at = 0, own_at = 0;
  // (notes of a call that gave up are old ones, or none)
  auto pieces = [&](int first, int last) {
    if (first >= 0 && first <= last && last < T.workers) return last - first + 1;
    set_status(A.status, ST_INTERNAL);
    return 0;
  };
  // A CTA that gave up on a wait (it has set the status) leaves notes and slots as an older call left them: nothing of this call is
  // to be used, and every row says so with NaN.  (Asked for here, used at the end: nothing waits for it.)
  const uint2 gave_up = reinterpret_cast<const uint2*>(T.gave_up)[lane];
  const int with_pre = *T.plan, pre0 = T.pre_first[pre_unit], pre1 = T.pre_last[pre_unit], own0 = T.own_first[own_unit], own1 = T.own_last[own_unit];
  const bool own = own_keys(T, attend_len(A, b, false)).tiles > 0;
  if (with_pre > 0) {
    n_pre = pieces(pre0, pre1);
    pre_at = (pre_unit + pre0) * pre_step + pre_row;
  }
  if (own) {
    n_own = pieces(own0, own1);
    own_at = (own_unit + own0) * own_step + own_row;
  }
  const int n = n_pre + n_own;
  auto lse_of = [&](int p) { return p < n_pre ? T.pre_lse[pre_at + p * pre_step] : T.own_lse[own_at + (p - n_pre) * own_step]; };
  constexpr int E = D / 32;
  auto load = [&](int p, float (&o)[E]) {
    const float* src = (p < n_pre ? T.pre_o + (pre_at + p * pre_step) * D : T.own_o + (own_at + (p - n_pre) * own_step) * D) + lane * E;
    if (E == 4) *reinterpret_cast<float4*>(o) = *reinterpret_cast<const float4*>(src);
    else *reinterpret_cast<float2*>(o) = *reinterpret_cast<const float2*>(src);
  };
  // the outputs of this warp's first pieces are asked for together with the weights
  constexpr int AHEAD = 4;
  float o[AHEAD][E], acc[E] = {}, tot = 0.f, top = -INFINITY;
#pragma unroll
  for (int k = 0; k < AHEAD; ++k)
    if (part + k * WARPS < n) load(part + k * WARPS, o[k]);
  for (int p = lane; p < n; p += 32) top = fmaxf(top, lse_of(p));
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  for (int p0 = 0; p0 < n; p0 += 32) {
    const float e = p0 + lane < n ? lse_of(p0 + lane) : -INFINITY;
    const float wl = e == -INFINITY ? 0.f : ex2(e - top);
    tot += warp_sum(wl);
    // (a piece that saw nothing has no output: its place may hold anything)
    const int m = min(32, n - p0);
    for (int j = part; j < m; j += AHEAD * WARPS) {
      if (p0 + j != part) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
          if (j + k * WARPS < m) load(p0 + j + k * WARPS, o[k]);
      }
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const float w = __shfl_sync(0xffffffffu, wl, (j + k * WARPS) & 31);
        if (j + k * WARPS < m && w != 0.f) {
#pragma unroll
          for (int c = 0; c < E; ++c) acc[c] = fmaf(w, o[k][c], acc[c]);
        }
      }
    }
  }
  const bool broken = __any_sync(0xffffffffu, (gave_up.x | gave_up.y) != 0);
  const float inv = broken ? NAN : tot == 0.f ? 0.f : 1.f / tot;
  uint16_t* dst = static_cast<uint16_t*>(A.out) + t * A.out_stride + (long long)hd * D;
  if (lane == 0 && part == 0 && A.lse) A.lse[row] = broken ? NAN : tot == 0.f ? -INFINITY : (top + log2f(tot)) * LN2;
  if (WARPS > 1) {
#pragma unroll
    for (int c = 0; c < E; ++c) s_acc[warp][lane * E + c] = acc[c];
    __syncthreads();
    const int c = threadIdx.x;
    if (c < D) {
      float o = 0.f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) o += s_acc[w][c];
      dst[c] = narrow16<WD>(o * inv);
    }
    return;
  }
#pragma unroll
  for (int c = 0; c < E; c += 2) {
    const uint32_t v = pack2<WD>(acc[c] * inv, acc[c + 1] * inv);
    if ((A.out_stride & 1) == 0 && (reinterpret_cast<uintptr_t>(A.out) & 3) == 0) reinterpret_cast<uint32_t*>(dst + lane * E)[c / 2] = v;
    else { dst[lane * E + c] = (uint16_t)v; dst[lane * E + c + 1] = (uint16_t)(v >> 16); }
  }
}

}  // namespace ls
