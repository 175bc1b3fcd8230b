// Host side of the attention half of a decoder layer: ls_paged_kv_*, ls_block_norm (argument checks, workspaces, launches).
#include "../../include/leanstream.h"

#include <algorithm>
#include <new>
#include <utility>

#include "ls_append.cuh"
#include "ls_attend.cuh"
#include "ls_attend_tile.cuh"
#include "ls_host.cuh"
#include "ls_norm.cuh"

using namespace ls_host;

struct ls_paged_kv {
  ls_paged_kv_desc d{};
  int sm_count = 148;
  float* part_o = nullptr;    // workspace of ls_attend_rows_kernel
  float* part_lse = nullptr;
  int* status = nullptr;
  // the tile kernels, where the pages can be copied as boxes
  bool tiles = false;
  int box = 0;
  CUtensorMap map_k{}, map_v{};
  size_t pre_slots = 0, own_slots = 0, own_units = 0, pre_units = 0;  // in rows, rows, units, units
  float* tile_ws = nullptr;
  int32_t* tile_ids = nullptr;
};

namespace {

// Blocks that ls_attend_rows_kernel is split into when rows are few: eight blocks of four warps per SM.
constexpr int kRowsBlocks = 148 * 8;
constexpr int kRowsMaxGroup = 8;
// Rows of a norm from which on threads take more of a row each (four blocks to an SM): 2000 x 4096 18.3 us with two chunks a thread
// against 23.0 with one, 64 x 4096 2.8 with one against 3.0; 8192 x 256 4.9 us with a warp per row against 8.9 with a block.
// Odd widths from half as many on: 300 x 1001 3.2 us with eight elements a thread against 4.7 with one, 64 x 1001 2.3 with one
// against 2.7.
constexpr int kNormManyRows = 148 * 4;
// Up to this many output rows the pieces of each are joined by eight warps (all blocks are resident at once), else by one.
constexpr long long kJoinFewRows = 148 * 8;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Each pointer (NULL among them) lies at a multiple of its element's `size` bytes: the kernels' accesses would fault otherwise.
template <class... P>
bool elements_aligned(size_t size, P... p) {
  return ((reinterpret_cast<uintptr_t>(p) | ...) & (size - 1)) == 0;
}

void free_kv(ls_paged_kv* kv) {
  cudaFree(kv->part_o); cudaFree(kv->part_lse); cudaFree(kv->status); cudaFree(kv->tile_ws); cudaFree(kv->tile_ids);
  delete kv;
}

// How the rows of n_seqs sequences of q_len tokens are cut into tiles, and what workspace the cut needs.
struct TileCut {
  int tq, tb, ts, rt, pairs;
  size_t pre_rows, own_rows, pre_units, own_units;
  TileCut(int n_seqs, int q_len, int kv_heads, int group, int ctas) {
    const long long tokens = (long long)n_seqs * q_len;
    tq = 128 / group;
    tb = (int)std::min<long long>(tq, tokens);
    ts = std::min(tq, q_len);
    rt = (q_len + ts - 1) / ts;
    const long long tiles = (tokens + tq - 1) / tq;
    pairs = tiles > 1 ? (int)((tiles + 1) / 2) : 0;
    pre_units = (size_t)kv_heads * std::max(pairs, 1);
    own_units = (size_t)n_seqs * kv_heads * rt;
    pre_rows = pairs ? (pre_units + ctas) * 256 : (pre_units + 2 * ctas) * 128;
    own_rows = (own_units + 2 * ctas) * ts * group;
  }
};

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
std::atomic<EncodeFn> g_encode{nullptr};

int32_t encoder(EncodeFn* out) {
  EncodeFn f = g_encode.load(std::memory_order_acquire);
  if (!f) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    LS_CUDA(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q));
    if (!p || q != cudaDriverEntryPointSuccess) return fail(LS_ERR_CUDA, "cuTensorMapEncodeTiled is not available");
    f = reinterpret_cast<EncodeFn>(p);
    g_encode.store(f, std::memory_order_release);
  }
  *out = f;
  return LS_OK;
}

// A map of 16-bit elements whose boxes are 64 elements (128 bytes, swizzled) wide; strides in bytes of dimensions 1...
int32_t make_map(CUtensorMap* map, int dtype, void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  EncodeFn enc = nullptr;
  LS_TRY(encoder(&enc));
  const cuuint32_t one[5] = {1, 1, 1, 1, 1};
  const CUresult rc = enc(map, dtype == LS_WDTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, rank, base, dims, strides, box,
                          one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (rc != CUDA_SUCCESS) return fail(LS_ERR_CUDA, "cuTensorMapEncodeTiled: error %d", (int)rc);
  return LS_OK;
}

int32_t page_map(CUtensorMap* map, const ls_paged_kv_desc& d, void* base, int box) {
  const cuuint64_t dims[4] = {(cuuint64_t)d.head_dim, (cuuint64_t)d.page_size, (cuuint64_t)d.n_kv_heads, (cuuint64_t)d.n_pages};
  // (the stride of a dimension of one is never used; the pool's own may be anything)
  const cuuint64_t strides[3] = {(cuuint64_t)d.token_stride * 2, (cuuint64_t)(d.n_kv_heads > 1 ? d.head_stride : d.head_dim) * 2,
                                 (cuuint64_t)(d.n_pages > 1 ? d.page_stride : d.head_dim) * 2};
  const cuuint32_t boxes[4] = {64, (cuuint32_t)box, 1, 1};
  return make_map(map, d.dtype, base, 4, dims, strides, boxes);
}

// The tile kernels copy boxes of a page: head dimensions of whole 128-byte columns, pages of a multiple of eight tokens,
// everything 16-byte aligned, a group that fits a tile.
bool tiles_apply(const ls_paged_kv_desc& d) {
  const int64_t limit = 1LL << 38;
  auto good = [&](int64_t stride, int n) { return n == 1 || (stride >= 8 && stride % 8 == 0 && stride < limit); };
  return (d.head_dim == 64 || d.head_dim == 128) && d.page_size % 8 == 0 && aligned16(d.d_k) && aligned16(d.d_v) && good(d.token_stride, d.page_size) &&
         good(d.head_stride, d.n_kv_heads) && good(d.page_stride, d.n_pages) && d.n_q_heads / d.n_kv_heads <= 128;
}

template <int WD, int D>
cudaError_t tile_attribute() {
  return cudaFuncSetAttribute(ls::ls_attend_tile_kernel<WD, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, ls::TileShape<D>::SMEM);
}

int32_t create_tiles(ls_paged_kv* kv) {
  const ls_paged_kv_desc& d = kv->d;
  kv->box = 8;
  while (kv->box < 128 && d.page_size % (kv->box * 2) == 0) kv->box *= 2;
  LS_TRY(page_map(&kv->map_k, d, d.d_k, kv->box));
  LS_TRY(page_map(&kv->map_v, d, d.d_v, kv->box));
  if (d.head_dim == 64) LS_CUDA((d.dtype == LS_WDTYPE_BF16 ? tile_attribute<ls::WD_BF16, 64>() : tile_attribute<ls::WD_FP16, 64>()));
  else LS_CUDA((d.dtype == LS_WDTYPE_BF16 ? tile_attribute<ls::WD_BF16, 128>() : tile_attribute<ls::WD_FP16, 128>()));
  const TileCut c(d.max_seqs, d.max_q_len, d.n_kv_heads, d.n_q_heads / d.n_kv_heads, kv->sm_count);
  // (fewer rows may need more pieces when they fit a single tile)
  kv->pre_slots = std::max(c.pre_rows, (size_t)(d.n_kv_heads + 2 * kv->sm_count) * 128);
  kv->own_slots = c.own_rows;
  kv->pre_units = c.pre_units;
  kv->own_units = c.own_units;
  LS_TRY(dalloc(&kv->tile_ws, (kv->pre_slots + kv->own_slots) * (d.head_dim + 1)));
  const size_t ids = ls::AT_MAX_CTAS / 4 + 2 * (kv->pre_units + kv->own_units) + 1;
  LS_TRY(dalloc(&kv->tile_ids, ids));
  LS_CUDA(cudaMemset(kv->tile_ids, 0, ids * sizeof(int32_t)));
  kv->tiles = true;
  return LS_OK;
}

// Launches that may start while the kernel in front of them ends; the kernels wait for it before they touch memory.
template <class... P, class... Q>
int32_t launch_early(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, Q&&... args) {
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  LS_CUDA(cudaLaunchKernelEx(&cfg, kernel, std::forward<Q>(args)...));
  LS_LAUNCHED();
  return LS_OK;
}

template <int WD, int D>
int32_t attend_tiles(ls_paged_kv* kv, const ls::AttendArgs& a, cudaStream_t st) {
  ls::TileArgs t{};
  t.a = a;
  const TileCut c(a.n_seqs, a.q_len, a.kv_heads, a.group, kv->sm_count);
  if (c.pre_rows > kv->pre_slots || c.own_rows > kv->own_slots || c.pre_units > kv->pre_units || c.own_units > kv->own_units)
    return fail(LS_ERR_INTERNAL, "ls_paged_kv_attend: workspace");
  t.tq = c.tq; t.tb = c.tb; t.ts = c.ts; t.rt = c.rt; t.pairs = c.pairs; t.box = kv->box;
  t.pre_o = kv->tile_ws; t.own_o = t.pre_o + kv->pre_slots * D;
  t.pre_lse = t.own_o + kv->own_slots * D; t.own_lse = t.pre_lse + kv->pre_slots;
  t.gave_up = reinterpret_cast<uint8_t*>(kv->tile_ids);
  t.pre_first = kv->tile_ids + ls::AT_MAX_CTAS / 4; t.pre_last = t.pre_first + kv->pre_units;
  t.own_first = t.pre_last + kv->pre_units; t.own_last = t.own_first + kv->own_units;
  t.plan = t.own_last + kv->own_units;
  t.workers = 2 * kv->sm_count;
  CUtensorMap q_all, q_own;
  const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)a.heads, (cuuint64_t)a.n_seqs * a.q_len};
  const cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)a.q_stride * 2};
  const cuuint32_t box_all[3] = {64, (cuuint32_t)a.group, (cuuint32_t)c.tb}, box_own[3] = {64, (cuuint32_t)a.group, (cuuint32_t)c.ts};
  void* q = const_cast<void*>(a.q);
  LS_TRY(make_map(&q_own, WD == ls::WD_BF16 ? LS_WDTYPE_BF16 : LS_WDTYPE_FP16, q, 3, dims, strides, box_own));
  if (a.prefix > 0) LS_TRY(make_map(&q_all, WD == ls::WD_BF16 ? LS_WDTYPE_BF16 : LS_WDTYPE_FP16, q, 3, dims, strides, box_all));
  else q_all = q_own;
  LS_TRY(launch_early(ls::ls_attend_tile_kernel<WD, D>, dim3((unsigned)kv->sm_count), ls::AT_THREADS, ls::TileShape<D>::SMEM, st, t, kv->map_k, kv->map_v,
                      q_all, q_own));
  const long long rows = (long long)a.n_seqs * a.q_len * a.heads;
  if (rows <= kJoinFewRows) return launch_early(ls::ls_attend_tile_join_kernel<WD, D, 8>, dim3((unsigned)rows), 256, 0, st, t);
  return launch_early(ls::ls_attend_tile_join_kernel<WD, D, 1>, dim3((unsigned)((rows + 7) / 8)), 256, 0, st, t);
}

int32_t create_kv(ls_paged_kv* kv) {
  const ls_paged_kv_desc& d = kv->d;
  int sms = 0;
  LS_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, d.device));
  kv->sm_count = sms;
  LS_TRY(dalloc(&kv->status, 1));
  LS_CUDA(cudaMemset(kv->status, 0, sizeof(int)));
  if (d.max_seqs > 0) {
    const size_t rows = (size_t)kRowsBlocks * kRowsMaxGroup;
    LS_TRY(dalloc(&kv->part_o, rows * d.head_dim));
    LS_TRY(dalloc(&kv->part_lse, rows));
    if (tiles_apply(d) && sms <= ls::AT_MAX_CTAS) LS_TRY(create_tiles(kv));
  }
  // (the clearing above runs on the default stream, which other streams need not wait for)
  LS_CUDA(cudaStreamSynchronize(nullptr));
  return LS_OK;
}

template <int WD, int NG>
int32_t launch_rows(const ls::AttendArgs& a, int lpk, int vec, cudaStream_t st) {
  const long long blocks = (long long)a.n_seqs * a.q_len * a.kv_heads * ((a.group + NG - 1) / NG) * a.splits;
  ls::ls_attend_rows_kernel<WD, NG><<<(unsigned)blocks, ls::AR_THREADS, 4 * NG * (a.dim + 2) * sizeof(float), st>>>(a, lpk, vec);
  LS_LAUNCHED();
  return LS_OK;
}

template <int WD>
int32_t attend_rows(ls::AttendArgs& a, bool q_vec, cudaStream_t st) {
  const int ng = a.group == 1 ? 1 : a.group <= 4 ? 4 : 8;
  const long long one = (long long)a.n_seqs * a.q_len * a.kv_heads * ((a.group + ng - 1) / ng);
  a.splits = (int)std::max(1LL, std::min(64LL, kRowsBlocks / one));
  if (one * a.splits > 0x7fffffffLL) return fail(LS_ERR_INVALID, "ls_paged_kv_attend: too many rows");
  int lpk = 1;
  while (lpk * 8 < a.dim) lpk *= 2;
  const bool kv_vec = aligned16(a.k) && aligned16(a.v) && a.page_stride % 8 == 0 && a.token_stride % 8 == 0 && a.head_stride % 8 == 0;
  const int vec = (kv_vec ? 1 : 0) | (q_vec ? 2 : 0);
  if (ng == 1) LS_TRY((launch_rows<WD, 1>(a, lpk, vec, st)));
  else if (ng == 4) LS_TRY((launch_rows<WD, 4>(a, lpk, vec, st)));
  else LS_TRY((launch_rows<WD, 8>(a, lpk, vec, st)));
  if (a.splits > 1) {
    const long long rows = (long long)a.n_seqs * a.q_len * a.heads;
    ls::ls_attend_rows_join_kernel<WD><<<(unsigned)((rows + 7) / 8), 256, 0, st>>>(a);
    LS_LAUNCHED();
  }
  return LS_OK;
}

template <int XT, int BT, int V, int K>
int32_t norm_blocks(const ls::NormArgs& a, cudaStream_t st) {
  const int chunks = a.d / V, threads = ((chunks + K - 1) / K + 31) / 32 * 32;
  return launch_early(ls::ls_norm_kernel<XT, BT, V, K, false>, dim3((unsigned)a.n), threads, 0, st, a);
}
template <int XT, int BT, int V, int K>
int32_t norm_warps(const ls::NormArgs& a, cudaStream_t st) {
  return launch_early(ls::ls_norm_kernel<XT, BT, V, K, true>, dim3((unsigned)((a.n + 7) / 8)), 256, 0, st, a);
}

template <int XT, int BT>
int32_t launch_norm(const ls::NormArgs& a, cudaStream_t st) {
  auto fits = [](const void* p, int64_t stride, bool rows) { return !p || (aligned16(p) && (!rows || stride % 8 == 0)); };
  const bool rows = a.n > 1;
  const bool vec = a.d % 8 == 0 && fits(a.x, a.x_stride, rows) && fits(a.y, a.y_stride, rows) && fits(a.x_out, a.x_out_stride, rows) &&
                   fits(a.h, a.h_stride, rows) && fits(a.gate, a.gate_stride, rows) && fits(a.w_post, 0, false) && fits(a.w_pre, 0, false);
  // Few rows are spread over as many threads as they have chunks; many rows take more per thread, so that fewer threads wait for
  // a row's sums, and short ones a warp each.
  if (vec) {
    const int chunks = a.d / 8;
    if (a.n >= kNormManyRows && chunks <= 32) return norm_warps<XT, BT, 8, 1>(a, st);
    if (a.n >= kNormManyRows && chunks <= 64) return norm_warps<XT, BT, 8, 2>(a, st);
    if (chunks <= 256 || (a.n < kNormManyRows && chunks <= 1024)) return norm_blocks<XT, BT, 8, 1>(a, st);
    return norm_blocks<XT, BT, 8, 2>(a, st);
  }
  if (a.n >= kNormManyRows / 2) {
    if (a.d <= 256) return norm_warps<XT, BT, 1, 8>(a, st);
    if (a.d <= 4096) return norm_blocks<XT, BT, 1, 8>(a, st);
    return norm_blocks<XT, BT, 1, 16>(a, st);
  }
  if (a.d <= 1024) return norm_blocks<XT, BT, 1, 1>(a, st);
  if (a.d <= 4096) return norm_blocks<XT, BT, 1, 4>(a, st);
  if (a.d <= 8192) return norm_blocks<XT, BT, 1, 8>(a, st);
  return norm_blocks<XT, BT, 1, 16>(a, st);
}

}  // namespace

extern "C" {

int32_t ls_paged_kv_create(const ls_paged_kv_desc* D, ls_paged_kv** out) {
  if (out) *out = nullptr;
  if (!D || !out) return fail(LS_ERR_INVALID, "ls_paged_kv_create: NULL argument");
  if (D->struct_size != sizeof(ls_paged_kv_desc))
    return fail(LS_ERR_INVALID, "ls_paged_kv_create: struct_size %u, expected %zu", D->struct_size, sizeof(ls_paged_kv_desc));
  if (D->dtype != LS_WDTYPE_BF16 && D->dtype != LS_WDTYPE_FP16) return fail(LS_ERR_INVALID, "ls_paged_kv_create: unknown dtype");
  if (D->n_kv_heads < 1 || D->n_q_heads < 1 || D->n_q_heads % D->n_kv_heads || D->n_q_heads > 65536)
    return fail(LS_ERR_INVALID, "ls_paged_kv_create: n_q_heads must be a positive multiple of n_kv_heads");
  if (D->head_dim < 8 || D->head_dim % 8 || D->head_dim > 256)
    return fail(LS_ERR_INVALID, "ls_paged_kv_create: head_dim must be a multiple of 8 in [8, 256]");
  if (D->page_size < 1 || D->n_pages < 1) return fail(LS_ERR_INVALID, "ls_paged_kv_create: page_size and n_pages must be positive");
  if (!D->d_k || !D->d_v) return fail(LS_ERR_INVALID, "ls_paged_kv_create: missing pages");
  if ((reinterpret_cast<uintptr_t>(D->d_k) | reinterpret_cast<uintptr_t>(D->d_v)) & 1)
    return fail(LS_ERR_INVALID, "ls_paged_kv_create: misaligned pages");
  if (D->page_stride < 0 || D->token_stride < 0 || D->head_stride < 0) return fail(LS_ERR_INVALID, "ls_paged_kv_create: negative stride");
  if (D->max_seqs < 0 || D->max_q_len < 0 || (D->max_seqs > 0) != (D->max_q_len > 0))
    return fail(LS_ERR_INVALID, "ls_paged_kv_create: max_seqs and max_q_len must both be positive, or both 0");
  if (D->d_rope && (D->rope_dim < 2 || D->rope_dim % 2 || D->rope_dim > D->head_dim || D->rope_positions < 1))
    return fail(LS_ERR_INVALID, "ls_paged_kv_create: rope_dim must be even in [2, head_dim] and rope_positions positive");
  if (D->d_rope && (reinterpret_cast<uintptr_t>(D->d_rope) & 3)) return fail(LS_ERR_INVALID, "ls_paged_kv_create: misaligned rotation table");
  int ndev = 0;
  LS_CUDA(cudaGetDeviceCount(&ndev));
  if (D->device < 0 || D->device >= ndev) return fail(LS_ERR_INVALID, "device %d out of range", D->device);
  DeviceGuard guard(D->device);
  ls_paged_kv* kv = new (std::nothrow) ls_paged_kv();
  if (!kv) return fail(LS_ERR_NOMEM, "host allocation");
  kv->d = *D;
  if (!D->d_rope) kv->d.rope_dim = kv->d.rope_positions = 0;
  const int32_t rc = create_kv(kv);
  if (rc != LS_OK) {
    free_kv(kv);  // (leaves the error's text alone)
    cudaGetLastError();
    return rc;
  }
  *out = kv;
  return LS_OK;
}

int32_t ls_paged_kv_destroy(ls_paged_kv* kv) {
  if (!kv) return LS_OK;
  DeviceGuard guard(kv->d.device);
  cudaDeviceSynchronize();
  free_kv(kv);
  return LS_OK;
}

int32_t ls_paged_kv_status(ls_paged_kv* kv, int32_t* host_status) {
  if (!kv || !host_status) return fail(LS_ERR_INVALID, "ls_paged_kv_status: NULL argument");
  DeviceGuard guard(kv->d.device);
  LS_CUDA(cudaDeviceSynchronize());
  int v = 0;
  LS_CUDA(cudaMemcpy(&v, kv->status, sizeof v, cudaMemcpyDeviceToHost));
  LS_CUDA(cudaMemset(kv->status, 0, sizeof v));
  LS_CUDA(cudaStreamSynchronize(nullptr));  // (a later call on a stream that does not wait for the default one may report something)
  *host_status = v;
  return LS_OK;
}

int32_t ls_paged_kv_append(ls_paged_kv* kv, const void* d_q, int64_t q_stride, void* d_q_out, int64_t q_out_stride, const void* d_k,
                           int64_t k_stride, const void* d_v, int64_t v_stride, int32_t n_tokens, const int32_t* d_seq,
                           const int32_t* d_pos, const int32_t* d_table, int32_t n_seqs, int32_t table_width, int64_t table_stride,
                           void* stream) {
  if (!kv) return fail(LS_ERR_INVALID, "ls_paged_kv_append: NULL handle");
  if (n_tokens < 0 || n_seqs < 0 || table_width < 0) return fail(LS_ERR_INVALID, "ls_paged_kv_append: negative size");
  if (n_tokens == 0) return LS_OK;
  if (!d_k || !d_v || !d_seq || !d_pos || (!d_table && n_seqs > 0 && table_width > 0))
    return fail(LS_ERR_INVALID, "ls_paged_kv_append: k, v, seq, pos and table are required");
  if ((d_q == nullptr) != (d_q_out == nullptr)) return fail(LS_ERR_INVALID, "ls_paged_kv_append: q and q_out go together");
  const ls_paged_kv_desc& D = kv->d;
  const int64_t qw = (int64_t)D.n_q_heads * D.head_dim, kw = (int64_t)D.n_kv_heads * D.head_dim;
  if (k_stride < kw || v_stride < kw || (d_q && (q_stride < qw || q_out_stride < qw)))
    return fail(LS_ERR_INVALID, "ls_paged_kv_append: a token stride is smaller than a token");
  if (n_seqs > 1 && table_stride < table_width) return fail(LS_ERR_INVALID, "ls_paged_kv_append: table_stride is smaller than table_width");
  if (!elements_aligned(2, d_q, d_q_out, d_k, d_v) || !elements_aligned(4, d_seq, d_pos, d_table))
    return fail(LS_ERR_INVALID, "ls_paged_kv_append: a misaligned pointer");
  DeviceGuard guard(D.device);
  ls::AppendArgs a{};
  a.q = static_cast<const uint16_t*>(d_q); a.q_out = static_cast<uint16_t*>(d_q_out);
  a.k = static_cast<const uint16_t*>(d_k); a.v = static_cast<const uint16_t*>(d_v);
  a.k_pages = static_cast<uint16_t*>(D.d_k); a.v_pages = static_cast<uint16_t*>(D.d_v);
  a.seq = d_seq; a.pos = d_pos; a.table = d_table; a.rope = D.d_rope; a.status = kv->status;
  a.q_stride = q_stride; a.q_out_stride = q_out_stride; a.k_stride = k_stride; a.v_stride = v_stride;
  a.page_stride = D.page_stride; a.token_stride = D.token_stride; a.head_stride = D.head_stride; a.table_stride = table_stride;
  a.n_tokens = n_tokens; a.n_seqs = n_seqs; a.heads = D.n_q_heads; a.kv_heads = D.n_kv_heads; a.dim = D.head_dim;
  a.page = D.page_size; a.n_pages = D.n_pages; a.table_width = table_width;
  a.rope_dim = D.rope_dim; a.rope_positions = D.rope_positions; a.interleaved = D.rope_interleaved;
  const cudaStream_t st = (cudaStream_t)stream;
  KernelTimer timer(LS_TIMED_APPEND, st);
  const bool bf = D.dtype == LS_WDTYPE_BF16;
  const bool vec = D.head_dim % 16 == 0 && D.rope_dim % 16 == 0 && aligned16(d_k) && aligned16(d_v) && aligned16(D.d_k) && aligned16(D.d_v) &&
                   aligned16(d_q) && aligned16(d_q_out) && aligned16(D.d_rope) &&
                   (n_tokens == 1 || (k_stride | v_stride | (d_q ? q_stride | q_out_stride : 0)) % 8 == 0) &&
                   (D.page_stride | D.token_stride | D.head_stride) % 8 == 0;
  if (vec) {
    // Two heads to a thread; where half a block or less is enough for that, a block holds several tokens (39785 tokens of 8 + 2 heads
    // of 64, most of a block idle otherwise, 118 us -> 22; the division by the width costs 80 heads of 128 a sixth, 118 -> 138).
    const int heads = (d_q ? D.n_q_heads : 0) + 2 * D.n_kv_heads, width = D.head_dim / 16 * ((heads + 1) / 2), per_block = std::max(1, 256 / width);
    if (per_block == 1)
      return launch_early(bf ? ls::ls_append_kernel<ls::WD_BF16, false> : ls::ls_append_kernel<ls::WD_FP16, false>, dim3((unsigned)n_tokens), 256, 0, st, a, 256);
    return launch_early(bf ? ls::ls_append_kernel<ls::WD_BF16, true> : ls::ls_append_kernel<ls::WD_FP16, true>,
                        dim3((unsigned)((n_tokens + per_block - 1) / per_block)), 256, 0, st, a, width);
  }
  const int items = ((d_q ? D.n_q_heads : 0) + 2 * D.n_kv_heads) * (D.head_dim / 2);
  const dim3 grid((unsigned)n_tokens, (unsigned)std::min(64, (items + 255) / 256));
  return launch_early(bf ? ls::ls_append_pairs_kernel<ls::WD_BF16> : ls::ls_append_pairs_kernel<ls::WD_FP16>, grid, 256, 0, st, a);
}

int32_t ls_paged_kv_attend(ls_paged_kv* kv, const void* d_q, int64_t q_stride, void* d_out, int64_t out_stride, float* d_lse,
                           int32_t n_seqs, int32_t q_len, const int32_t* d_seq_len, const int32_t* d_table, int32_t table_width,
                           int64_t table_stride, const int32_t* d_prefix_pages, int32_t prefix_len, int32_t window, float scale,
                           void* stream) {
  if (!kv) return fail(LS_ERR_INVALID, "ls_paged_kv_attend: NULL handle");
  if (n_seqs < 0 || q_len < 0 || table_width < 0 || prefix_len < 0 || window < 0)
    return fail(LS_ERR_INVALID, "ls_paged_kv_attend: negative size");
  const ls_paged_kv_desc& D = kv->d;
  if (n_seqs > D.max_seqs || q_len > D.max_q_len)
    return fail(LS_ERR_INVALID, "ls_paged_kv_attend: %d sequences of %d tokens, the handle was created for %d of %d", n_seqs, q_len, D.max_seqs,
                D.max_q_len);
  if (n_seqs == 0 || q_len == 0) return LS_OK;
  if (!d_q || !d_out || !d_seq_len || (!d_table && table_width > 0)) return fail(LS_ERR_INVALID, "ls_paged_kv_attend: q, out, seq_len and table are required");
  if (prefix_len > ls::MAX_POSITIONS) return fail(LS_ERR_INVALID, "ls_paged_kv_attend: prefix_len beyond %d positions", ls::MAX_POSITIONS);
  if (prefix_len > 0 && !d_prefix_pages) return fail(LS_ERR_INVALID, "ls_paged_kv_attend: prefix_len without prefix pages");
  const int64_t qw = (int64_t)D.n_q_heads * D.head_dim;
  if (q_stride < qw || out_stride < qw) return fail(LS_ERR_INVALID, "ls_paged_kv_attend: a token stride is smaller than a token");
  if (n_seqs > 1 && table_stride < table_width) return fail(LS_ERR_INVALID, "ls_paged_kv_attend: table_stride is smaller than table_width");
  if (!(scale > 0.f) || scale > 1e30f) return fail(LS_ERR_INVALID, "ls_paged_kv_attend: scale must be positive and finite");
  if (!elements_aligned(2, d_q, d_out) || !elements_aligned(4, d_lse, d_seq_len, d_table, d_prefix_pages))
    return fail(LS_ERR_INVALID, "ls_paged_kv_attend: a misaligned pointer");
  DeviceGuard guard(D.device);
  ls::AttendArgs a{};
  a.q = d_q; a.out = d_out; a.lse = d_lse; a.k = D.d_k; a.v = D.d_v; a.seq_len = d_seq_len; a.table = d_table; a.prefix_pages = d_prefix_pages;
  a.status = kv->status; a.part_o = kv->part_o; a.part_lse = kv->part_lse;
  a.q_stride = q_stride; a.out_stride = out_stride; a.page_stride = D.page_stride; a.token_stride = D.token_stride;
  a.head_stride = D.head_stride; a.table_stride = table_stride;
  a.n_seqs = n_seqs; a.q_len = q_len; a.heads = D.n_q_heads; a.kv_heads = D.n_kv_heads; a.group = D.n_q_heads / D.n_kv_heads; a.dim = D.head_dim;
  a.page = D.page_size; a.n_pages = D.n_pages; a.table_width = table_width; a.prefix = prefix_len; a.window = window;
  a.scale_log2 = scale * ls::LOG2E;
  const cudaStream_t st = (cudaStream_t)stream;
  KernelTimer timer(LS_TIMED_ATTEND, st);
  const bool q_vec = aligned16(d_q) && q_stride % 8 == 0;
  // The tile kernel counts the cost of (unit, tile) pairs, at most five each, in 31 bits; what could exceed that goes the other way.
  const double tiles = (double)D.n_kv_heads * (((double)n_seqs * q_len + 1) * (prefix_len / 128.0 + 2) + (double)n_seqs * q_len * ((double)table_width * D.page_size / 128 + 2));
  if (kv->tiles && q_vec && tiles < 4e8) {
    if (D.head_dim == 64) return D.dtype == LS_WDTYPE_BF16 ? attend_tiles<ls::WD_BF16, 64>(kv, a, st) : attend_tiles<ls::WD_FP16, 64>(kv, a, st);
    return D.dtype == LS_WDTYPE_BF16 ? attend_tiles<ls::WD_BF16, 128>(kv, a, st) : attend_tiles<ls::WD_FP16, 128>(kv, a, st);
  }
  return D.dtype == LS_WDTYPE_BF16 ? attend_rows<ls::WD_BF16>(a, q_vec, st) : attend_rows<ls::WD_FP16>(a, q_vec, st);
}

int32_t ls_block_norm(const void* d_x, int64_t x_stride, int32_t x_dtype, const void* d_y, int64_t y_stride, int32_t dtype, void* d_x_out,
                      int64_t x_out_stride, void* d_h, int64_t h_stride, int32_t n, int32_t d, int32_t post_norm, const float* d_w_post,
                      const void* d_gate, int64_t gate_stride, float scale, int32_t pre_norm, const float* d_w_pre, float eps,
                      void* stream) {
  if (n < 0 || d < 1 || d > 16384) return fail(LS_ERR_INVALID, "ls_block_norm: n must not be negative and d must be in [1, 16384]");
  if (dtype != LS_WDTYPE_BF16 && dtype != LS_WDTYPE_FP16 && dtype != LS_DTYPE_F32) return fail(LS_ERR_INVALID, "ls_block_norm: unknown dtype");
  if (x_dtype != LS_DTYPE_F32 && x_dtype != dtype) return fail(LS_ERR_INVALID, "ls_block_norm: the residual is float or of the block's type");
  if ((post_norm != LS_NORM_RMS && post_norm != LS_NORM_NONE) || (pre_norm != LS_NORM_RMS && pre_norm != LS_NORM_NONE))
    return fail(LS_ERR_INVALID, "ls_block_norm: unknown norm");
  if (!(eps >= 0.f)) return fail(LS_ERR_INVALID, "ls_block_norm: eps must not be negative");
  if (n == 0) return LS_OK;
  if (!d_x || (!d_x_out && !d_h)) return fail(LS_ERR_INVALID, "ls_block_norm: x and one of x_out, h are required");
  if (!d_y && (d_w_post || d_gate)) return fail(LS_ERR_INVALID, "ls_block_norm: a gain or gate of a block needs the block's output y");
  if (n > 1 && (x_stride < d || (d_y && y_stride < d) || (d_x_out && x_out_stride < d) || (d_h && h_stride < d) ||
                (d_gate && gate_stride != 0 && gate_stride < d)))
    return fail(LS_ERR_INVALID, "ls_block_norm: a row stride is smaller than a row");
  if (!elements_aligned(x_dtype == LS_DTYPE_F32 ? 4 : 2, d_x, d_x_out) ||
      !elements_aligned(dtype == LS_DTYPE_F32 ? 4 : 2, d_y, d_h, d_gate) || !elements_aligned(4, d_w_post, d_w_pre))
    return fail(LS_ERR_INVALID, "ls_block_norm: a misaligned pointer");
  int dev = -1;
  LS_CUDA(cudaGetDevice(&dev));
  static const int n_dev = [] { int k = 0; return cudaGetDeviceCount(&k) == cudaSuccess ? k : 0; }();
  if (n_dev > 1) {
    cudaPointerAttributes at{};
    if (cudaPointerGetAttributes(&at, d_x) == cudaSuccess && at.type == cudaMemoryTypeDevice) dev = at.device;
    else cudaGetLastError();
  }
  DeviceGuard guard(dev);
  ls::NormArgs a{};
  a.x = d_x; a.y = d_y; a.x_out = d_x_out; a.h = d_h; a.w_post = d_w_post; a.w_pre = d_w_pre; a.gate = d_gate;
  a.x_stride = x_stride; a.y_stride = y_stride; a.x_out_stride = x_out_stride; a.h_stride = h_stride; a.gate_stride = gate_stride;
  a.n = n; a.d = d; a.post = post_norm == LS_NORM_RMS; a.pre = pre_norm == LS_NORM_RMS; a.scale = scale; a.eps = eps;
  const cudaStream_t st = (cudaStream_t)stream;
  KernelTimer timer(LS_TIMED_NORM, st);
  if (x_dtype == LS_DTYPE_F32) {
    if (dtype == LS_WDTYPE_BF16) return launch_norm<ls::DT_F32, ls::WD_BF16>(a, st);
    if (dtype == LS_WDTYPE_FP16) return launch_norm<ls::DT_F32, ls::WD_FP16>(a, st);
    return launch_norm<ls::DT_F32, ls::DT_F32>(a, st);
  }
  return dtype == LS_WDTYPE_BF16 ? launch_norm<ls::WD_BF16, ls::WD_BF16>(a, st) : launch_norm<ls::WD_FP16, ls::WD_FP16>(a, st);
}

}  // extern "C"
