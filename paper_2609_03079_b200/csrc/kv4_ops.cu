// Host side of the 4-bit paged cache: ls_paged_kv4_* (argument checks, workspaces, launches).
#include "../../include/leanstream.h"

#include <algorithm>
#include <new>

#include "ls_host.cuh"
#include "ls_kv4.cuh"
#include "ls_kv4_shapes.cuh"

using namespace ls_host;

struct ls_paged_kv4 {
  ls_paged_kv4_desc d{};
  int sm_count = 148;
  int* status = nullptr;
  float* part = nullptr;       // workspace of the attention
  int32_t* arrived = nullptr;
  size_t part_floats = 0, units = 0;
  uint16_t* q = nullptr;       // queries that do not lie at a multiple of 16 bytes are copied here
};

namespace {

using ls_kv4::Shape;

// Rows of queries of one key head: 8 or 16 at a time (8 with heads of 256, whose sums fill the registers), or so few that 8 columns
// hold each row for each group.
Shape shape_for(const ls_paged_kv4_desc& d, long long rows) {
  const int groups = d.head_dim / d.group, nt = groups > 1 && rows * groups <= 8 ? 0 : rows <= 8 || d.head_dim == 256 ? 1 : 2;
  return d.dtype == LS_WDTYPE_BF16 ? ls_kv4::shape_bf16(d.head_dim, d.group, nt) : ls_kv4::shape_fp16(d.head_dim, d.group, nt);
}

ls::FastDiv fast_div(int d) {
  uint32_t up = 0;
  while ((1u << up) < (uint32_t)d) ++up;
  return {(uint32_t)(((1ULL << (31 + up)) + d - 1) / d), 31 + up};
}

void free_kv(ls_paged_kv4* kv) {
  cudaFree(kv->part); cudaFree(kv->q); cudaFree(kv->arrived); cudaFree(kv->status);
  delete kv;
}

int32_t create_kv(ls_paged_kv4* kv) {
  const ls_paged_kv4_desc& d = kv->d;
  LS_CUDA(cudaDeviceGetAttribute(&kv->sm_count, cudaDevAttrMultiProcessorCount, d.device));
  LS_TRY(dalloc(&kv->status, 1));
  LS_CUDA(cudaMemset(kv->status, 0, sizeof(int)));
  if (d.max_seqs > 0) {
    const long long rows = (long long)d.max_q_len * (d.n_q_heads / d.n_kv_heads);
    for (long long r : {1LL, 8LL, 16LL}) {  // (one of each shape that so many rows can have)
      const Shape s = shape_for(d, std::min(r, rows));
      LS_CUDA(cudaFuncSetAttribute(s.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, s.smem));
      kv->part_floats = std::max(kv->part_floats, (size_t)kv->sm_count * (s.threads / 32) * 2 * s.piece);
      kv->units = std::max(kv->units, (size_t)d.max_seqs * d.n_kv_heads * ((size_t)(rows + s.rows - 1) / s.rows));
    }
    LS_TRY(dalloc(&kv->part, kv->part_floats));
    LS_TRY(dalloc(&kv->q, (size_t)d.max_seqs * d.max_q_len * d.n_q_heads * d.head_dim));
    LS_TRY(dalloc(&kv->arrived, kv->units));
    LS_CUDA(cudaMemset(kv->arrived, 0, kv->units * sizeof(int32_t)));
  }
  // (the clearing above runs on the default stream, which other streams need not wait for)
  LS_CUDA(cudaStreamSynchronize(nullptr));
  return LS_OK;
}

int32_t check_table(const char* what, const int32_t* d_table, int32_t n_seqs, int32_t table_width, int64_t table_stride) {
  if (n_seqs < 0 || table_width < 0) return fail(LS_ERR_INVALID, "%s: negative size", what);
  if (!d_table && n_seqs > 0 && table_width > 0) return fail(LS_ERR_INVALID, "%s: the table is required", what);
  if (n_seqs > 1 && table_stride < table_width) return fail(LS_ERR_INVALID, "%s: table_stride is smaller than table_width", what);
  if (!elements_aligned(4, d_table)) return fail(LS_ERR_INVALID, "%s: a misaligned pointer", what);
  return LS_OK;
}

ls::Kv4Pages pages_of(const ls_paged_kv4* kv, const int32_t* d_table, int32_t n_seqs, int32_t table_width, int64_t table_stride) {
  const ls_paged_kv4_desc& D = kv->d;
  ls::Kv4Pages p{};
  p.pages = static_cast<uint8_t*>(D.d_pages); p.table = d_table; p.status = kv->status;
  p.page_stride = D.page_stride; p.head_stride = D.head_stride; p.table_stride = table_stride;
  p.n_seqs = n_seqs; p.kv_heads = D.n_kv_heads; p.group = D.group; p.page = D.page_size; p.n_pages = D.n_pages; p.table_width = table_width;
  return p;
}

using AppendKernel = void (*)(ls::Kv4AppendArgs);
template <int WD, int D>
AppendKernel append_of_group(int group) {
  if (group == 32) return ls::ls_kv4_append_kernel<WD, D, 32>;
  if constexpr (D >= 128) {
    if (group == 128) return ls::ls_kv4_append_kernel<WD, D, 128>;
  }
  return ls::ls_kv4_append_kernel<WD, D, 64>;
}
template <int WD>
AppendKernel append_kernel(int dim, int group) {
  return dim == 64 ? append_of_group<WD, 64>(group) : dim == 128 ? append_of_group<WD, 128>(group) : append_of_group<WD, 256>(group);
}
template <int WD>
auto read_kernel(int dim) {
  return dim == 64 ? ls::ls_kv4_read_kernel<WD, 64> : dim == 128 ? ls::ls_kv4_read_kernel<WD, 128> : ls::ls_kv4_read_kernel<WD, 256>;
}

}  // namespace

extern "C" {

int64_t ls_paged_kv4_block_bytes(int32_t page_size, int32_t head_dim, int32_t group) {
  if (head_dim != 64 && head_dim != 128 && head_dim != 256) return fail(LS_ERR_INVALID, "ls_paged_kv4: head_dim must be 64, 128 or 256");
  if ((group != 32 && group != 64 && group != 128) || group > head_dim) return fail(LS_ERR_INVALID, "ls_paged_kv4: group must be 32, 64 or 128, at most head_dim");
  if (page_size < 16 || page_size % 16) return fail(LS_ERR_INVALID, "ls_paged_kv4: page_size must be a positive multiple of 16");
  return (int64_t)(page_size / 16) * ls::kv4_tile(head_dim, group);
}

int32_t ls_paged_kv4_create(const ls_paged_kv4_desc* D, ls_paged_kv4** out) {
  if (out) *out = nullptr;
  if (!D || !out) return fail(LS_ERR_INVALID, "ls_paged_kv4_create: NULL argument");
  if (D->struct_size != sizeof(ls_paged_kv4_desc))
    return fail(LS_ERR_INVALID, "ls_paged_kv4_create: struct_size %u, expected %zu", D->struct_size, sizeof(ls_paged_kv4_desc));
  if (D->dtype != LS_WDTYPE_BF16 && D->dtype != LS_WDTYPE_FP16) return fail(LS_ERR_INVALID, "ls_paged_kv4_create: unknown dtype");
  if (D->n_kv_heads < 1 || D->n_q_heads < 1 || D->n_q_heads % D->n_kv_heads || D->n_q_heads > 65536)
    return fail(LS_ERR_INVALID, "ls_paged_kv4_create: n_q_heads must be a positive multiple of n_kv_heads");
  const int64_t block = ls_paged_kv4_block_bytes(D->page_size, D->head_dim, D->group);
  if (block < 0) return LS_ERR_INVALID;
  if (D->n_pages < 1) return fail(LS_ERR_INVALID, "ls_paged_kv4_create: n_pages must be positive");
  if (!D->d_pages) return fail(LS_ERR_INVALID, "ls_paged_kv4_create: missing pages");
  if (!aligned16(D->d_pages)) return fail(LS_ERR_INVALID, "ls_paged_kv4_create: misaligned pages");
  if ((D->n_pages > 1 && (D->page_stride < block || D->page_stride % 16)) || (D->n_kv_heads > 1 && (D->head_stride < block || D->head_stride % 16)))
    return fail(LS_ERR_INVALID, "ls_paged_kv4_create: a stride is smaller than a block or no multiple of 16 bytes");
  if (D->max_seqs < 0 || D->max_q_len < 0 || (D->max_seqs > 0) != (D->max_q_len > 0))
    return fail(LS_ERR_INVALID, "ls_paged_kv4_create: max_seqs and max_q_len must both be positive, or both 0");
  // (rows and units are counted in 32 bits)
  if ((double)D->max_seqs * D->max_q_len * D->n_q_heads > 1e9) return fail(LS_ERR_INVALID, "ls_paged_kv4_create: max_seqs * max_q_len is too large");
  if (D->d_rope && (D->rope_dim < 2 || D->rope_dim % 2 || D->rope_dim > D->head_dim || D->rope_positions < 1))
    return fail(LS_ERR_INVALID, "ls_paged_kv4_create: rope_dim must be even in [2, head_dim] and rope_positions positive");
  if (!elements_aligned(4, D->d_rope)) return fail(LS_ERR_INVALID, "ls_paged_kv4_create: misaligned rotation table");
  int ndev = 0;
  LS_CUDA(cudaGetDeviceCount(&ndev));
  if (D->device < 0 || D->device >= ndev) return fail(LS_ERR_INVALID, "device %d out of range", D->device);
  DeviceGuard guard(D->device);
  ls_paged_kv4* kv = new (std::nothrow) ls_paged_kv4();
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

int32_t ls_paged_kv4_destroy(ls_paged_kv4* kv) {
  if (!kv) return LS_OK;
  DeviceGuard guard(kv->d.device);
  cudaDeviceSynchronize();
  free_kv(kv);
  return LS_OK;
}

int32_t ls_paged_kv4_status(ls_paged_kv4* kv, int32_t* host_status) {
  if (!kv || !host_status) return fail(LS_ERR_INVALID, "ls_paged_kv4_status: NULL argument");
  DeviceGuard guard(kv->d.device);
  LS_CUDA(cudaDeviceSynchronize());
  int v = 0;
  LS_CUDA(cudaMemcpy(&v, kv->status, sizeof v, cudaMemcpyDeviceToHost));
  LS_CUDA(cudaMemset(kv->status, 0, sizeof v));
  LS_CUDA(cudaStreamSynchronize(nullptr));  // (a later call on a stream that does not wait for the default one may report something)
  *host_status = v;
  return LS_OK;
}

int32_t ls_paged_kv4_append(ls_paged_kv4* kv, const void* d_q, int64_t q_stride, void* d_q_out, int64_t q_out_stride, const void* d_k,
                            int64_t k_stride, const void* d_v, int64_t v_stride, int32_t n_tokens, const int32_t* d_seq,
                            const int32_t* d_pos, const int32_t* d_table, int32_t n_seqs, int32_t table_width, int64_t table_stride,
                            void* stream) {
  if (!kv) return fail(LS_ERR_INVALID, "ls_paged_kv4_append: NULL handle");
  if (n_tokens < 0) return fail(LS_ERR_INVALID, "ls_paged_kv4_append: negative size");
  LS_TRY(check_table("ls_paged_kv4_append", d_table, n_seqs, table_width, table_stride));
  if (n_tokens == 0) return LS_OK;
  if (!d_k || !d_v || !d_seq || !d_pos) return fail(LS_ERR_INVALID, "ls_paged_kv4_append: k, v, seq and pos are required");
  if ((d_q == nullptr) != (d_q_out == nullptr)) return fail(LS_ERR_INVALID, "ls_paged_kv4_append: q and q_out go together");
  const ls_paged_kv4_desc& D = kv->d;
  const int64_t qw = (int64_t)D.n_q_heads * D.head_dim, kw = (int64_t)D.n_kv_heads * D.head_dim;
  if (k_stride < kw || v_stride < kw || (d_q && (q_stride < qw || q_out_stride < qw)))
    return fail(LS_ERR_INVALID, "ls_paged_kv4_append: a token stride is smaller than a token");
  if (!elements_aligned(2, d_q, d_q_out, d_k, d_v) || !elements_aligned(4, d_seq, d_pos)) return fail(LS_ERR_INVALID, "ls_paged_kv4_append: a misaligned pointer");
  DeviceGuard guard(D.device);
  ls::Kv4AppendArgs a{};
  a.p = pages_of(kv, d_table, n_seqs, table_width, table_stride);
  a.q = static_cast<const uint16_t*>(d_q); a.q_out = static_cast<uint16_t*>(d_q_out);
  a.k = static_cast<const uint16_t*>(d_k); a.v = static_cast<const uint16_t*>(d_v);
  a.seq = d_seq; a.pos = d_pos; a.rope = D.d_rope;
  a.q_stride = q_stride; a.q_out_stride = q_out_stride; a.k_stride = k_stride; a.v_stride = v_stride;
  a.n_tokens = n_tokens; a.heads = D.n_q_heads; a.rope_dim = D.rope_dim; a.rope_positions = D.rope_positions; a.interleaved = D.rope_interleaved;
  const bool one = n_tokens == 1;
  a.kv_vec = aligned16(d_k) && aligned16(d_v) && (one || (k_stride | v_stride) % 8 == 0);
  a.q_vec = D.rope_dim % 16 == 0 && aligned16(d_q) && aligned16(d_q_out) && aligned16(D.d_rope) && (one || !d_q || (q_stride | q_out_stride) % 8 == 0);
  a.rope_vec = D.rope_dim % 16 == 0 && aligned16(D.d_rope);
  const int64_t kv_job = 256 * ls::K4_SLABS, q_job = 512 * ls::K4_Q_HEADS;
  a.kv_jobs = (int)((kw + kv_job - 1) / kv_job);
  a.jobs = 2 * a.kv_jobs + (d_q ? (int)((qw + q_job - 1) / q_job) : 0);
  const unsigned long long blocks = ((unsigned long long)n_tokens * a.jobs + 7) / 8;
  if (blocks > 0x1fffffffULL) return fail(LS_ERR_INVALID, "ls_paged_kv4_append: too many tokens");
  const cudaStream_t st = (cudaStream_t)stream;
  KernelTimer timer(LS_TIMED_APPEND4, st);
  return launch_early(D.dtype == LS_WDTYPE_BF16 ? append_kernel<ls::WD_BF16>(D.head_dim, D.group) : append_kernel<ls::WD_FP16>(D.head_dim, D.group), dim3((unsigned)blocks), 256, 0, st, a);
}

int32_t ls_paged_kv4_attend(ls_paged_kv4* kv, const void* d_q, int64_t q_stride, void* d_out, int64_t out_stride, float* d_lse,
                            int32_t n_seqs, int32_t q_len, const int32_t* d_seq_len, const int32_t* d_table, int32_t table_width,
                            int64_t table_stride, int32_t window, float scale, void* stream) {
  if (!kv) return fail(LS_ERR_INVALID, "ls_paged_kv4_attend: NULL handle");
  if (q_len < 0 || window < 0) return fail(LS_ERR_INVALID, "ls_paged_kv4_attend: negative size");
  LS_TRY(check_table("ls_paged_kv4_attend", d_table, n_seqs, table_width, table_stride));
  const ls_paged_kv4_desc& D = kv->d;
  if (n_seqs > D.max_seqs || q_len > D.max_q_len)
    return fail(LS_ERR_INVALID, "ls_paged_kv4_attend: %d sequences of %d tokens, the handle was created for %d of %d", n_seqs, q_len, D.max_seqs,
                D.max_q_len);
  if (n_seqs == 0 || q_len == 0) return LS_OK;
  if (!d_q || !d_out || !d_seq_len) return fail(LS_ERR_INVALID, "ls_paged_kv4_attend: q, out and seq_len are required");
  const int64_t qw = (int64_t)D.n_q_heads * D.head_dim;
  if (q_stride < qw || out_stride < qw) return fail(LS_ERR_INVALID, "ls_paged_kv4_attend: a token stride is smaller than a token");
  if (!(scale > 0.f) || scale > 1e30f) return fail(LS_ERR_INVALID, "ls_paged_kv4_attend: scale must be positive and finite");
  if (!elements_aligned(2, d_q, d_out) || !elements_aligned(4, d_lse, d_seq_len)) return fail(LS_ERR_INVALID, "ls_paged_kv4_attend: a misaligned pointer");
  DeviceGuard guard(D.device);
  const long long rows = (long long)q_len * (D.n_q_heads / D.n_kv_heads);
  const Shape s = shape_for(D, rows);
  const long long row_tiles = (rows + s.rows - 1) / s.rows, per_seq = row_tiles * D.n_kv_heads;
  if ((size_t)n_seqs * per_seq > kv->units || (size_t)kv->sm_count * (s.threads / 32) * 2 * s.piece > kv->part_floats)
    return fail(LS_ERR_INTERNAL, "ls_paged_kv4_attend: workspace");
  // A launch counts its tiles in 32 bits: of as many sequences as cannot have too many (all of them but for huge tables).
  // (64: more than what a unit's beginning counts for)
  const long long most = per_seq * (64 + std::min((long long)table_width * D.page_size, (long long)ls::MAX_POSITIONS) / 16);
  if (most > ls::K4_MAX_BLOCKS) return fail(LS_ERR_INVALID, "ls_paged_kv4_attend: q_len * table_width is too large");
  const int32_t step = (int32_t)std::min<long long>(n_seqs, ls::K4_MAX_BLOCKS / most);
  const cudaStream_t st = (cudaStream_t)stream;
  KernelTimer timer(LS_TIMED_ATTEND4, st);
  if (!aligned16(d_q) || (n_seqs * (long long)q_len > 1 && q_stride % 8)) {
    LS_TRY(launch_early(ls::ls_kv4_align_kernel<256>, dim3((unsigned)(n_seqs * q_len)), 256, 0, st, static_cast<const uint16_t*>(d_q), q_stride, kv->q, (int)qw));
    d_q = kv->q;
    q_stride = qw;
  }
  for (int32_t b = 0; b < n_seqs; b += step) {
    ls::Attend4Args a{};
    const long long tokens = (long long)b * q_len;
    a.p = pages_of(kv, d_table ? d_table + b * table_stride : nullptr, std::min(step, n_seqs - b), table_width, table_stride);
    a.q = static_cast<const uint16_t*>(d_q) + tokens * q_stride; a.out = static_cast<uint16_t*>(d_out) + tokens * out_stride;
    a.lse = d_lse ? d_lse + tokens * D.n_q_heads : nullptr; a.seq_len = d_seq_len + b;
    a.part = kv->part; a.arrived = kv->arrived;
    a.q_stride = q_stride; a.out_stride = out_stride;
    a.q_len = q_len; a.heads = D.n_q_heads; a.group = D.n_q_heads / D.n_kv_heads; a.window = window ? window : 0x7fffffff;
    a.row_tiles = (int)row_tiles;
    a.most = (int)std::min((long long)table_width * D.page_size, (long long)ls::MAX_POSITIONS);
    a.behind = (int)std::min<long long>(0x7fffffff, (long long)a.window + q_len - 1);
    a.by_group = fast_div(a.group); a.by_row_tiles = fast_div(a.row_tiles); a.by_page = fast_div(D.page_size / 16);
    a.out_vec = (reinterpret_cast<uintptr_t>(d_out) & 7) == 0 && (n_seqs * (long long)q_len == 1 || out_stride % 4 == 0);
    a.scale_log2 = scale * ls::LOG2E;
    LS_TRY(launch_early(s.kernel, dim3((unsigned)kv->sm_count), s.threads, s.smem, st, a));
  }
  return LS_OK;
}

int32_t ls_paged_kv4_read(ls_paged_kv4* kv, void* d_k_out, int64_t k_stride, void* d_v_out, int64_t v_stride, int32_t n_tokens,
                          const int32_t* d_seq, const int32_t* d_pos, const int32_t* d_table, int32_t n_seqs, int32_t table_width,
                          int64_t table_stride, void* stream) {
  if (!kv) return fail(LS_ERR_INVALID, "ls_paged_kv4_read: NULL handle");
  if (n_tokens < 0) return fail(LS_ERR_INVALID, "ls_paged_kv4_read: negative size");
  LS_TRY(check_table("ls_paged_kv4_read", d_table, n_seqs, table_width, table_stride));
  if (n_tokens == 0) return LS_OK;
  if ((!d_k_out && !d_v_out) || !d_seq || !d_pos) return fail(LS_ERR_INVALID, "ls_paged_kv4_read: seq, pos and one of k_out, v_out are required");
  const ls_paged_kv4_desc& D = kv->d;
  const int64_t kw = (int64_t)D.n_kv_heads * D.head_dim;
  if ((d_k_out && k_stride < kw) || (d_v_out && v_stride < kw)) return fail(LS_ERR_INVALID, "ls_paged_kv4_read: a token stride is smaller than a token");
  if (!elements_aligned(2, d_k_out, d_v_out) || !elements_aligned(4, d_seq, d_pos)) return fail(LS_ERR_INVALID, "ls_paged_kv4_read: a misaligned pointer");
  DeviceGuard guard(D.device);
  ls::Kv4ReadArgs a{};
  a.p = pages_of(kv, d_table, n_seqs, table_width, table_stride);
  a.k = static_cast<uint16_t*>(d_k_out); a.v = static_cast<uint16_t*>(d_v_out); a.seq = d_seq; a.pos = d_pos;
  a.k_stride = k_stride; a.v_stride = v_stride; a.n_tokens = n_tokens;
  a.vec = aligned16(d_k_out) && aligned16(d_v_out) && (n_tokens == 1 || ((d_k_out ? k_stride : 0) | (d_v_out ? v_stride : 0)) % 8 == 0);
  // Threads of a token: half of its pieces each, or a fraction that leaves fewer of a block's threads idle.  (33 and 36 heads of 128: 88 and 81 us, by halves
  // alone 96 and 90; 7 of 256: 180 and 189; 40 of 128, 4092 tokens: 27 and 26.)
  const int items = D.n_kv_heads * (D.head_dim / 16);
  auto busy = [](int width) { return 256 / width * width; };
  a.width = std::min(256, (items + 1) / 2);
  for (int part = 3; part <= 6; ++part)
    if (busy((items + part - 1) / part) > busy(a.width) + 16) a.width = (items + part - 1) / part;
  const int per_block = 256 / a.width;
  const cudaStream_t st = (cudaStream_t)stream;
  KernelTimer timer(LS_TIMED_READ4, st);
  return launch_early(D.dtype == LS_WDTYPE_BF16 ? read_kernel<ls::WD_BF16>(D.head_dim) : read_kernel<ls::WD_FP16>(D.head_dim),
                      dim3((unsigned)((n_tokens + (long long)per_block - 1) / per_block)), 256, 0, st, a);
}

}  // extern "C"
