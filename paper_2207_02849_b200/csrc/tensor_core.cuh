// Building blocks of the persistent tensor-core kernels (grouped.cu, vocab_products.cu): instruction wrappers, tensor maps and
// aligned copies of operands.
#pragma once
#include <cuda.h>
#include "common.cuh"

namespace betty {
namespace tc {

static constexpr int BM = 128;                // accumulator lanes of one CTA
static constexpr int BK = 64;                 // contraction chunk: 64 operand values = one 128-byte swizzle row
static constexpr int A_BYTES = BM * BK * 2;
static constexpr uint32_t SPIN = 1u << 24;

// ------------------------------------------------------------------ instruction wrappers
__device__ __forceinline__ uint32_t s_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint64_t* bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(s_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void expect_tx(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(s_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool try_wait(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(ok) : "r"(s_u32(bar)), "r"(parity) : "memory");
  return ok != 0;
}
// bounded; gives up early once another role has
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  for (uint32_t i = 0; i < SPIN; ++i) {
    if (try_wait(bar, parity)) return true;
    if ((i & 1023u) == 1023u && *abort_flag) return false;
  }
  *abort_flag = 1;
  return false;
}
__device__ __forceinline__ uint32_t in_cta(uint32_t smem_addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* tm) { asm volatile("prefetch.tensormap [%0];" ::"l"(tm) : "memory"); }
template <int CG>
__device__ __forceinline__ void load_2d(void* dst, const CUtensorMap* tm, int x, int y, uint32_t bar) {
  if (CG == 1)
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(s_u32(dst)), "l"(tm), "r"(x), "r"(y), "r"(bar) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(s_u32(dst)), "l"(tm), "r"(x), "r"(y), "r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ void load_3d(void* dst, const CUtensorMap* tm, int x, int y, int z, uint32_t bar) {
  if (CG == 1)
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(s_u32(dst)), "l"(tm), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(s_u32(dst)), "l"(tm), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ void load_4d(void* dst, const CUtensorMap* tm, int x, int y, int z, int w, uint32_t bar) {
  if (CG == 1)
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(s_u32(dst)), "l"(tm), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(s_u32(dst)), "l"(tm), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}
// shared-memory matrix descriptor, 128-byte swizzle: start address, leading and stride byte offsets in 16-byte units
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lbo, uint32_t sbo) {
  return (uint64_t)((addr >> 4) & 0x3FFF) | (uint64_t)((lbo >> 4) & 0x3FFF) << 16 | (uint64_t)((sbo >> 4) & 0x3FFF) << 32 |
         (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
template <int CG>
__device__ __forceinline__ void mma(uint32_t acc, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate) {
  if (CG == 1)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(acc), "l"(da), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(acc), "l"(da), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
}
// arrival on the barrier at this offset (in both CTAs of a pair) once the products issued so far are done
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar) {
  if (CG == 1)
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t (&r)[32], uint32_t taddr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr) : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// One lane of a converged warp, the same each time.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
  return p != 0;
}
// a value all lanes have, in a form the compiler knows to be the same for all
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }

template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f(float v) { return __float2half_rn(v); }

// ------------------------------------------------------------------ host side
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static inline EncodeTiledFn lookup_encode_fn() {
  void* p = nullptr;
  cudaDriverEntryPointQueryResult q;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess)
    return (EncodeTiledFn)p;
  (void)cudaGetLastError();
  return nullptr;
}
static inline EncodeTiledFn encode_fn() {
  static const EncodeTiledFn fn = lookup_encode_fn();
  return fn;
}

// an operand as the kernels read it: [groups][rows][cols], 16-bit values
struct Operand { const void* p; int64_t cols, rows, groups, ld, group_stride; };

static inline bool encode(CUtensorMap* tm, int dtype, int rank, const Operand& o, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  EncodeTiledFn fn = encode_fn();
  const cuuint32_t ones[4] = {1, 1, 1, 1};
  return fn && fn(tm, dtype == BETTY_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, (void*)o.p, dims, strides, box,
                  ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
static inline bool make_map(CUtensorMap* tm, int dtype, const Operand& o, bool three, int box_cols, int box_rows) {
  const cuuint64_t dims[3] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows, (cuuint64_t)o.groups};
  const cuuint64_t strides[2] = {(cuuint64_t)o.ld * 2, (cuuint64_t)o.group_stride * 2};
  const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1};
  return encode(tm, dtype, three ? 3 : 2, o, dims, strides, box);
}
// The same operand with its columns cut into blocks of 64 (their number a dimension of its own), so that one copy brings two
// blocks of 64 rows in the order that an MN-major operand wants: the issuing thread, not the bytes, bounds the loads
// otherwise.  Needs a multiple of 64 columns: a short last block would be read past its row.
static inline bool make_blocked_map(CUtensorMap* tm, int dtype, const Operand& o, bool three) {
  const cuuint64_t dims[4] = {64, (cuuint64_t)o.rows, (cuuint64_t)o.cols / 64, (cuuint64_t)o.groups};
  const cuuint64_t strides[3] = {(cuuint64_t)o.ld * 2, 128, (cuuint64_t)o.group_stride * 2};
  const cuuint32_t box[4] = {64, 64, 2, 1};
  return encode(tm, dtype, three ? 4 : 3, o, dims, strides, box);
}

static inline int64_t pad8(int64_t v) { return (v + 7) / 8 * 8; }

// The values c .. c + 7 of a row of 16-bit values (c a multiple of 8), zeros behind its last, never outside the row: of a row that starts on
// an 8-byte or 4-byte boundary as words of that size, of others the two 16-byte words around them, shifted together; the ends value
// by value, each in a word of its own.  In two steps, so that the words of several accesses are under way together.
struct Words { uint4 x, y; };
__device__ __forceinline__ int before_word(const uint16_t* row) { return (int)((uintptr_t)row & 15) >> 1; }   // values between a 16-byte boundary and the row
// whether whole words are read for c .. c + 7
__device__ __forceinline__ bool inside(int c, int cols, int m) { return m & 1 ? c >= m && c - m + 16 <= cols : c + 8 <= cols; }
__device__ __forceinline__ Words fetch8(const uint16_t* row, int c, int cols) {
  Words r = {make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
  const int m = before_word(row);
  if (inside(c, cols, m)) {
    if (m & 1) {
      r.x = *(const uint4*)(row + c - m);
      r.y = *(const uint4*)(row + c - m + 8);
    } else if (m & 2) {
      const uint32_t* p = (const uint32_t*)(row + c);
      r.x = make_uint4(p[0], p[1], p[2], p[3]);
    } else {
      const uint2 a = *(const uint2*)(row + c), b = *(const uint2*)(row + c + 4);
      r.x = make_uint4(a.x, a.y, b.x, b.y);
    }
  } else if (c < cols) {
    r.x.x = row[c];
    if (c + 1 < cols) r.x.y = row[c + 1];
    if (c + 2 < cols) r.x.z = row[c + 2];
    if (c + 3 < cols) r.x.w = row[c + 3];
    if (c + 4 < cols) r.y.x = row[c + 4];
    if (c + 5 < cols) r.y.y = row[c + 5];
    if (c + 6 < cols) r.y.z = row[c + 6];
    if (c + 7 < cols) r.y.w = row[c + 7];
  }
  return r;
}
__device__ __forceinline__ uint4 shift8(const Words& r, const uint16_t* row, int c, int cols) {
  const int m = before_word(row);
  if (!inside(c, cols, m)) return make_uint4(r.x.x | r.x.y << 16, r.x.z | r.x.w << 16, r.y.x | r.y.y << 16, r.y.z | r.y.w << 16);
  if (!(m & 1)) return r.x;
  uint32_t w[8] = {r.x.x, r.x.y, r.x.z, r.x.w, r.y.x, r.y.y, r.y.z, r.y.w};
#pragma unroll
  for (int k = 0; k < 6; ++k) w[k] = m & 4 ? w[k + 2] : w[k];
#pragma unroll
  for (int k = 0; k < 5; ++k) w[k] = m & 2 ? w[k + 1] : w[k];
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = __funnelshift_r(w[k], w[k + 1], 16);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Copies a [rows, cols] matrix of 16-bit values to rows of `ld` values (a multiple of 8, from a 16-byte boundary), which is
// what TMA reads; used for operands whose own rows do not start on 16-byte boundaries.  A warp takes a row at a time and a lane
// eight values, U accesses under way together (pieces of rows shared evenly among the lanes, or four segments of any
// rows at a time, took 157 and 174 us with their divisions where this takes 132).  Blocks of 256 threads.
struct AlignRows {
  const uint16_t* src; int64_t ld_src, rows_per_group, group_stride, rows; int cols;
  uint16_t* dst; int ld;
};
template <int U>
__device__ __forceinline__ void align_rows(const AlignRows& a, int64_t block, int64_t blocks) {
  const int lane = threadIdx.x & 31, cols = a.cols, ld = a.ld;
  for (int64_t row = block * 8 + (threadIdx.x >> 5); row < a.rows; row += blocks * 8) {
    const uint16_t* p = a.rows_per_group == a.rows ? a.src + row * a.ld_src
                                                   : a.src + (row / a.rows_per_group) * a.group_stride + (row % a.rows_per_group) * a.ld_src;
    uint16_t* q = a.dst + row * ld;
    for (int c0 = lane * 8; c0 < ld; c0 += 256 * U) {
      Words v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = fetch8(p, c0 + 256 * u, cols);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c0 + 256 * u < ld) *(uint4*)(q + c0 + 256 * u) = shift8(v[u], p, c0 + 256 * u, cols);
    }
  }
}

// The operand itself, or its rows copied to 16-byte boundaries in the workspace (align.cu).
betty_status align_operand(cudaStream_t stream, Arena& arena, Operand& o);
// The same without the launch: o becomes the copy that align_rows(a) still has to make (a.rows == 0: none).
betty_status plan_alignment(Arena& arena, Operand& o, AlignRows& a);
int64_t align_blocks(const AlignRows& a);

}  // namespace tc
}  // namespace betty
