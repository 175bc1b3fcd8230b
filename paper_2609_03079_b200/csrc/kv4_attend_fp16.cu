// The 4-bit attention kernels for fp16.
#include "ls_kv4_shapes.cuh"

namespace ls_kv4 {
Shape shape_fp16(int dim, int group, int nt) { return shape_of<ls::WD_FP16>(dim, group, nt); }
}  // namespace ls_kv4
