// The 4-bit attention kernels for bf16.
#include "ls_kv4_shapes.cuh"

namespace ls_kv4 {
Shape shape_bf16(int dim, int group, int nt) { return shape_of<ls::WD_BF16>(dim, group, nt); }
}  // namespace ls_kv4
