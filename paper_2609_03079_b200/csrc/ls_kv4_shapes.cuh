// The shapes of the 4-bit attention kernel, compiled in two files (one for each type) that build side by side.
#pragma once
#include "ls_kv4_attend.cuh"

namespace ls_kv4 {

struct Shape {
  void (*kernel)(ls::Attend4Args);
  int rows, threads, smem;
  size_t piece;  // floats
};
Shape shape_bf16(int dim, int group, int nt);
Shape shape_fp16(int dim, int group, int nt);

template <int WD, int D, int G, int NT>
Shape shape() {
  if constexpr (NT == 0 && D == G) return {};  // (one group: columns are rows)
  else {
  using S = ls::K4Shape<D, G, NT>;
  return {ls::ls_kv4_attend_kernel<WD, D, G, NT>, S::ROWS, S::THREADS, S::SMEM, S::PIECE / sizeof(float)};
  }
}
template <int WD, int D, int NT>
Shape shape_of_group(int group) {
  if (group == 32) return shape<WD, D, 32, NT>();
  if constexpr (D >= 128) {
    if (group == 128) return shape<WD, D, 128, NT>();
  }
  return shape<WD, D, 64, NT>();
}
template <int WD>
Shape shape_of(int dim, int group, int nt) {
  if (nt == 0) return dim == 64 ? shape_of_group<WD, 64, 0>(group) : dim == 128 ? shape_of_group<WD, 128, 0>(group) : shape_of_group<WD, 256, 0>(group);
  if (dim == 64) return nt == 1 ? shape_of_group<WD, 64, 1>(group) : shape_of_group<WD, 64, 2>(group);
  if (dim == 128) return nt == 1 ? shape_of_group<WD, 128, 1>(group) : shape_of_group<WD, 128, 2>(group);
  return shape_of_group<WD, 256, 1>(group);
}

}  // namespace ls_kv4
