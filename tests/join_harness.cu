// The second kernel of tiled attention alone, on a workspace made by hand: one row of one head, one piece.
#include "ls_attend_tile.cuh"

extern "C" int run_join(int few_rows, void* out, float* lse, float* part_o, float* part_lse, int* ids, int* seq_len, int* table, int* status, int ctas) {
  ls::TileArgs t{};
  t.a.out = out; t.a.lse = lse; t.a.seq_len = seq_len; t.a.table = table; t.a.status = status;
  t.a.out_stride = 64; t.a.table_stride = 1; t.a.table_width = 1;
  t.a.n_seqs = t.a.q_len = t.a.heads = t.a.kv_heads = t.a.group = 1;
  t.a.dim = 64; t.a.page = 16; t.a.n_pages = 1;
  t.tq = 128; t.tb = t.ts = t.rt = 1; t.box = 16;
  t.pre_o = t.own_o = part_o; t.pre_lse = t.own_lse = part_lse;
  t.pre_first = ids + 64; t.pre_last = ids + 65; t.own_first = ids + 66; t.own_last = ids + 67; t.plan = ids + 68;
  t.gave_up = reinterpret_cast<uint8_t*>(ids);
  t.workers = 2 * ctas;
  if (few_rows) ls::ls_attend_tile_join_kernel<ls::WD_BF16, 64, 8><<<1, 256>>>(t);
  else ls::ls_attend_tile_join_kernel<ls::WD_BF16, 64, 1><<<1, 256>>>(t);
  const cudaError_t rc = cudaGetLastError();
  return rc != cudaSuccess ? (int)rc : (int)cudaDeviceSynchronize();
}
