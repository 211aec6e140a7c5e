// Aligned copies of matrix operands whose rows TMA cannot read in place.
#include "tensor_core.cuh"

namespace betty {
namespace tc {

// Accesses a lane and blocks an SM: four and four; of narrow rows, which leave many of four unused, fewer accesses and more rows at a time.
// In us with U = 2 / 3 / 4: 40000 x 515 18.6 / 18.6 / 20.3, 30000 x 1030 22.9 / 24.7 / 24.2, 28056 x 1196 25.7 / 24.7 / 26.8, 8208 x 2052
// 16.4 / 14.8 / 14.5, 85056 x 2461 133.5 / 131.8 / 131.2 (836 MB, 6.4 TB/s).
template <int U>
__global__ void __launch_bounds__(256, 8 - U) k_align_rows(const AlignRows a) {
  pdl_enter();
  align_rows<U>(a, blockIdx.x, gridDim.x);
}

// The operand itself, or its rows copied to 16-byte boundaries in the workspace.
betty_status align_operand(cudaStream_t stream, Arena& arena, Operand& o) {
  AlignRows a;
  BETTY_TRY(plan_alignment(arena, o, a));
  if (!a.rows) return BETTY_OK;
  launch_pdl(a.ld <= 1088 ? k_align_rows<2> : (a.ld <= 1280 ? k_align_rows<3> : k_align_rows<4>), dim3((unsigned)align_blocks(a)), dim3(256), 0, stream, a);
  BETTY_LAUNCH_CHECK();
  return BETTY_OK;
}

betty_status plan_alignment(Arena& arena, Operand& o, AlignRows& a) {
  a = {};
  if (o.rows == 1) o.ld = pad8(o.cols);          // strides that are never used still have to be valid ones
  if (o.groups == 1) o.group_stride = o.rows * o.ld;
  if (aligned16(o.p) && o.ld % 8 == 0 && o.group_stride % 8 == 0) return BETTY_OK;
  const int64_t ld = pad8(o.cols), rows = o.rows * o.groups;
  uint16_t* dst = arena.alloc<uint16_t>((size_t)(rows * ld));
  if (!dst) return BETTY_ERR_WORKSPACE;
  const bool even = o.group_stride == o.rows * o.ld;        // one matrix of all groups' rows
  a = {(const uint16_t*)o.p, o.ld, even ? rows : o.rows, o.group_stride, rows, (int)o.cols, dst, (int)ld};
  o.p = dst; o.ld = ld; o.group_stride = o.rows * ld;
  return BETTY_OK;
}

int64_t align_blocks(const AlignRows& a) {
  const int64_t blocks = (a.rows + 7) / 8, most = (int64_t)current_sm_count() * 32;
  return blocks < most ? blocks : most;
}

}  // namespace tc
}  // namespace betty
