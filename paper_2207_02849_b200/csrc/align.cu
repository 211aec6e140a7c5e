// Aligned copies of matrix operands whose rows TMA cannot read in place.
#include "tensor_core.cuh"

namespace betty {
namespace tc {

__global__ void __launch_bounds__(256) k_align_rows(const AlignRows a) {
  pdl_enter();
  align_rows(a, blockIdx.x, gridDim.x);
}

// The operand itself, or its rows copied to 16-byte boundaries in the workspace.
betty_status align_operand(cudaStream_t stream, Arena& arena, Operand& o) {
  AlignRows a;
  BETTY_TRY(plan_alignment(arena, o, a));
  if (!a.rows) return BETTY_OK;
  launch_pdl(k_align_rows, dim3((unsigned)align_blocks(a)), dim3(256), 0, stream, a);
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
