// Aligned copies of matrix operands whose rows TMA cannot read in place.
#include "tensor_core.cuh"

namespace betty {
namespace tc {

// Copies a [rows, cols] matrix of 16-bit values to rows of `ld` values (a multiple of 8, from a 16-byte boundary), which is
// what TMA reads; used for operands whose own rows do not start on 16-byte boundaries.  A warp takes a row at a time and a lane
// four values: as 32-bit words where the row starts on a 4-byte boundary, else as the words around them, shifted together
// (never outside the row: its ends go value by value).
__global__ void __launch_bounds__(256) k_align_rows(const uint16_t* src, int64_t ld_src, int64_t rows_per_group, int64_t group_stride, int64_t rows,
                                                    int cols, uint16_t* dst, int ld) {
  pdl_enter();
  const int lane = threadIdx.x & 31;
  constexpr int U = 4;
  for (int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); row < rows; row += (int64_t)gridDim.x * 8) {
    const uint16_t* p = rows_per_group == rows ? src + row * ld_src : src + (row / rows_per_group) * group_stride + (row % rows_per_group) * ld_src;
    uint16_t* q = dst + row * ld;
    const bool odd = (uintptr_t)p & 2;
    for (int c0 = lane * 4; c0 < ld; c0 += 128 * U) {
      uint2 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + 128 * u;
        v[u] = make_uint2(0u, 0u);
        if (!odd && c + 4 <= cols) {
          v[u] = make_uint2(*(const uint32_t*)(p + c), *(const uint32_t*)(p + c + 2));
        } else if (odd && c > 0 && c + 5 <= cols) {
          const uint32_t a = *(const uint32_t*)(p + c - 1), b = *(const uint32_t*)(p + c + 1), d = *(const uint32_t*)(p + c + 3);
          v[u] = make_uint2(__funnelshift_r(a, b, 16), __funnelshift_r(b, d, 16));
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (c + k < cols) (k < 2 ? v[u].x : v[u].y) |= (uint32_t)p[c + k] << (16 * (k & 1));
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c0 + 128 * u < ld) *(uint2*)(q + c0 + 128 * u) = v[u];
    }
  }
}

// The operand itself, or its rows copied to 16-byte boundaries in the workspace.
betty_status align_operand(cudaStream_t stream, Arena& arena, Operand& o) {
  if (o.rows == 1) o.ld = pad8(o.cols);          // strides that are never used still have to be valid ones
  if (o.groups == 1) o.group_stride = o.rows * o.ld;
  if (aligned16(o.p) && o.ld % 8 == 0 && o.group_stride % 8 == 0) return BETTY_OK;
  const int64_t ld = pad8(o.cols), rows = o.rows * o.groups;
  uint16_t* dst = arena.alloc<uint16_t>((size_t)(rows * ld));
  if (!dst) return BETTY_ERR_WORKSPACE;
  const int64_t blocks = (rows + 7) / 8, most = (int64_t)current_sm_count() * 32;
  const bool even = o.group_stride == o.rows * o.ld;        // one matrix of all groups' rows
  launch_pdl(k_align_rows, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, stream, (const uint16_t*)o.p, o.ld,
             even ? rows : o.rows, o.group_stride, rows, (int)o.cols, dst, (int)ld);
  BETTY_LAUNCH_CHECK();
  o.p = dst; o.ld = ld; o.group_stride = o.rows * ld;
  return BETTY_OK;
}

}  // namespace tc
}  // namespace betty
