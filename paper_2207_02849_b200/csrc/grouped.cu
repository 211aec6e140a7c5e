// Matrix products grouped by expert: rows offsets[e] .. offsets[e+1]-1 of a batch belong to expert e with matrix W_e.
//
//   forward          Y_i  = W_e X_i            Y[i, o]    = sum_k X[i, k] W_e[o, k]
//   backward, data   dX_i = W_e^T dY_i         dX[i, k]   = sum_o dY[i, o] W_e[o, k]
//   backward, weight dW_e = sum_i dY_i X_i^T   dW_e[o, k] = sum over the expert's rows of dY[i, o] X[i, k]
//
// The offsets stay on the device: the host neither reads nor waits for them.  One persistent tcgen05 kernel serves all
// three: every CTA (or pair of CTAs) turns the offsets into the list of output tiles itself.  An accumulator holds the
// output's contiguous index in its lanes ("lane" dimension: o, k and k) and the other index in its columns (rows of the
// batch; o for the weight gradient), so that the ragged dimension of the first two products is the instruction's N: a
// tile takes any multiple of 16 (32 for a pair) rows up to its width, and an expert with few rows costs a narrow
// instruction, not an empty one.  In the weight gradient the ragged dimension is contracted over: the last chunk of an
// expert's rows must not read the next expert's, so the tensor maps of its operands end at the expert's last row and TMA
// fills the rest with zeros (k_group_maps writes one pair of maps per expert).
//
// Measured (bf16, alone with a cold L2 / back to back under the power cap): 16384 rows, 8 uneven experts, 4096 x 4096: 386 / 440 us,
// 1.42 / 1.25 PFLOP/s, 85 % of the measured library rate in both; weight gradient 4096 x 2048: 185 / 199 to 231 us (fp32 result 204 /
// 215).  5001 rows, 16 experts, 2048 -> 1024 (fp16): 29 us in a row, 33 among other passes, 39 alone with a cold L2, against 15 for its
// bytes.  Of that, 128 tiles on 74 pairs (two rounds, 1.73 would do) explain a sixth; the rest is the pace of about 320 ns per
// contraction chunk where one of 160 columns needs 230, the first loads and the last tiles' drain.
#include <cuda.h>
#include "common.cuh"

namespace betty {
namespace grouped {

enum Mode { FORWARD = 0, BACKWARD_DATA = 1, BACKWARD_WEIGHT = 2 };

static constexpr int BM = 128;                // accumulator lanes of one CTA
static constexpr int BK = 64;                 // contraction chunk: 64 operand values = one 128-byte swizzle row
static constexpr int A_BYTES = BM * BK * 2;
static constexpr int MAX_GROUPS = 1024;
static constexpr int THREADS = 320;           // warp 0: TMA, warp 1: MMA, warps 2-9: epilogue
static constexpr int EPI_WARPS = 8;
static constexpr uint32_t SPIN = 1u << 24;

template <int CG, int NT> struct Cfg {
  static constexpr int B_BYTES = NT / CG * BK * 2;          // each CTA of a pair stages half of the columns
  static_assert(NT / CG <= 128, "the boxes of B hold up to 128 columns of a CTA");
  static constexpr int STAGE = A_BYTES + B_BYTES;
  // narrow tiles leave room for the partial sums of a split contraction (SPLIT_BYTES for each CTA but the first)
  static constexpr int SPLIT_BYTES = NT <= 64 ? BM * NT * 4 : 0, MAX_SPLIT = NT <= 32 ? 4 : (NT <= 64 ? 2 : 1);
  static constexpr int STAGES = ((NT <= 64 ? 160 : 192) * 1024) / STAGE;
  static constexpr int TMEM_COLS = 2 * NT;                  // two accumulators: a tile drains while the next is multiplied
  static constexpr int smem(int groups, int split) { return STAGES * STAGE + 1024 + 256 + (split - 1) * SPLIT_BYTES + 2 * (groups + 1) * 4; }
};

struct Args {
  const int32_t* offsets;
  int groups, rows;
  int lanes;               // extent of the lane dimension
  int cols;                // BACKWARD_WEIGHT: extent of the column dimension
  int depth;               // contraction extent (not BACKWARD_WEIGHT)
  void* out; int64_t ldo, group_stride;
  uint32_t type_bits;      // operand format bits of the instruction descriptor
  int a_blocked, b_blocked;// MN-major operands: maps with 64-value blocks as a dimension of their own (see make_blocked_map)
  const CUtensorMap* maps; // BACKWARD_WEIGHT: [groups][2]
  int split;               // CTAs of a cluster that share a tile's contraction (single-SM tiles; then a cluster has one tile at most)
  StatusBlock* sb;
};

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

// ------------------------------------------------------------------ tiles
// Columns per tile of a group with n rows: the tiles of a group are of equal width, so that a few rows over a multiple of
// NT do not leave a nearly empty tile.
template <int CG, int NT>
__host__ __device__ __forceinline__ int tile_width(int n) {
  const int tiles = (n + NT - 1) / NT, step = 16 * CG;
  return (((n + tiles - 1) / tiles) + step - 1) / step * step;
}
// The offsets clamped to a non-decreasing sequence within [0, rows], and the number of tiles before each group; one warp.
// Values that had to be clamped are reported: every access stays in range whatever the caller passes.
template <int CG, int NT, int MODE>
__device__ __forceinline__ void list_tiles(const Args& a, int* off, int* before, bool report) {
  const int lane = threadIdx.x & 31, n = a.groups + 1, per = (n + 31) / 32;
  const int lane_tiles = (a.lanes + BM * CG - 1) / (BM * CG), col_tiles = (a.cols + NT - 1) / NT;
  const int i0 = lane * per, i1 = min(i0 + per, n);
  int top = 0;
  bool bad = false;
  for (int i = i0; i < i1; ++i) {
    const int v = a.offsets[i];
    bad |= v < 0 || v > a.rows || v < top || (i == 0 && v != 0);
    top = max(top, min(max(v, 0), a.rows));
    off[i] = i == 0 ? 0 : top;
  }
  int run = top;                                   // largest offset in this and the lanes before
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run = max(run, v);
  }
  const int prev = __shfl_up_sync(0xffffffffu, run, 1);
  if (lane > 0) {
    bad |= i0 < i1 && off[i0] < prev;
    for (int i = i0; i < i1; ++i) off[i] = max(off[i], prev);
  }
  if (__any_sync(0xffffffffu, bad) && lane == 0 && report) record_status(a.sb, BETTY_ERR_INVALID_ARG);
  __syncwarp();
  int sum = 0;
  for (int i = i0; i < i1 && i < a.groups; ++i) {
    const int rows = off[i + 1] - off[i];
    const int t = MODE == BACKWARD_WEIGHT ? col_tiles : (rows > 0 ? (rows + tile_width<CG, NT>(rows) - 1) / tile_width<CG, NT>(rows) : 0);
    before[i] = t * lane_tiles;
    sum += before[i];
  }
  int incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  int at = incl - sum;
  for (int i = i0; i < i1 && i < a.groups; ++i) { const int t = before[i]; before[i] = at; at += t; }
  if (lane == 31) before[a.groups] = incl;
  __syncwarp();
}

struct Tile {
  int group, chunks;       // contraction chunks; 0: nothing to multiply
  int l0, c0, width;       // first lane, first column, columns of the instruction
  int cols;                // columns to store
  int k0;                  // first contraction index (BACKWARD_WEIGHT: the group's first row)
};
// tile t; `group` is the caller's running position (tiles are taken in increasing order)
template <int CG, int NT, int MODE>
__device__ __forceinline__ Tile tile_at(const Args& a, const int* off, const int* before, int t, int& group) {
  while (t >= before[group + 1]) ++group;
  const int local = t - before[group], lane_tiles = (a.lanes + BM * CG - 1) / (BM * CG);
  const int row0 = off[group], rows = off[group + 1] - row0;
  Tile r;
  r.group = group;
  r.l0 = (local % lane_tiles) * (BM * CG);
  const int ct = local / lane_tiles;
  if (MODE == BACKWARD_WEIGHT) {
    r.c0 = ct * NT;
    r.cols = min(NT, a.cols - r.c0);
    r.width = r.cols > NT / 2 ? NT : NT / 2;       // operand blocks are 64 columns wide per CTA
    r.chunks = (rows + BK - 1) / BK;
    r.k0 = row0;
  } else {
    r.width = tile_width<CG, NT>(rows);
    r.c0 = row0 + ct * r.width;
    r.cols = min(r.width, row0 + rows - r.c0);
    r.chunks = (a.depth + BK - 1) / BK;
    r.k0 = 0;
  }
  return r;
}

template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f(float v) { return __float2half_rn(v); }

// the first n of 32 accumulator columns of this thread's lane
template <typename TO>
__device__ __forceinline__ void store_columns(TO* o, int64_t ldo, const uint32_t (&v)[32], int n) {
  if (n >= 32) {
#pragma unroll
    for (int k = 0; k < 32; ++k) o[k * ldo] = from_f<TO>(__uint_as_float(v[k]));
  } else {
#pragma unroll
    for (int k = 0; k < 32; ++k)
      if (k < n) o[k * ldo] = from_f<TO>(__uint_as_float(v[k]));
  }
}

// CG = 2: a pair of CTAs (a cluster of two) shares a tile of 256 lanes; each stages its own lanes of A and half of the
// columns of B, the even CTA issues the products, both hold the accumulator rows of their own lanes.
template <int CG, int NT, int MODE, typename TO>
__device__ __forceinline__ void body(const CUtensorMap& tmA, const CUtensorMap& tmB32, const CUtensorMap& tmB64, const CUtensorMap& tmB128, const Args& a) {
  using C = Cfg<CG, NT>;
  constexpr int S = C::STAGES;
  constexpr bool A_MN = MODE != FORWARD, B_MN = MODE == BACKWARD_WEIGHT;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint64_t* full = (uint64_t*)(smem + S * C::STAGE);
  uint64_t* empty = full + S;
  uint64_t* acc_full = empty + S;
  uint64_t* acc_empty = acc_full + 2;
  uint32_t* tmem_slot = (uint32_t*)(acc_empty + 2);
  volatile int* abort_flag = (volatile int*)(tmem_slot + 1);
  float* parts = (float*)(smem + S * C::STAGE + 256);        // split contraction: [CTA - 1][column][lane]
  int* off = (int*)((unsigned char*)parts + (a.split - 1) * C::SPLIT_BYTES);
  int* before = off + a.groups + 1;

  const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
  uint32_t rank = 0;
  const bool clustered = CG == 2 || a.split > 1;
  if (clustered) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  // a pair's rank is its half of the lanes; a split's rank is its part of the contraction
  const uint32_t half_rank = CG == 2 ? rank : 0;
  const int part_rank = CG == 1 ? (int)rank : 0;
  const int worker = blockIdx.x / (CG * a.split), workers = gridDim.x / (CG * a.split);

  if (tid == 0) {
    for (int s = 0; s < S; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(&acc_full[s], 1); mbar_init(&acc_empty[s], CG * EPI_WARPS); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    prefetch_map(&tmA); prefetch_map(&tmB32); prefetch_map(&tmB64); prefetch_map(&tmB128);
  }
  if (warp == 0) {
    if (CG == 1) {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(s_u32(tmem_slot)), "r"(C::TMEM_COLS) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(s_u32(tmem_slot)), "r"(C::TMEM_COLS) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
  }
  pdl_enter();             // global memory is touched from here on
  if (warp == 1) list_tiles<CG, NT, MODE>(a, off, before, blockIdx.x == 0);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (clustered) cluster_sync_all();   // the others' barriers exist before anything is signalled across the cluster
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem_base = *tmem_slot;
  const int tiles = before[a.groups];
  Tile mine = {};          // epilogue warps of a split: the cluster's tile
  int mine_l = 0;
  bool have_mine = false;

  // The loading and the multiplying warp run their loops with all lanes, and one lane issues: copies and products take their
  // descriptors and coordinates from uniform registers, and a loop that the compiler cannot see to be the same for the warp
  // moves each of them there one by one (measured: 400 ns per chunk of four products in a loop of lane 0 alone, whatever
  // their width, which was the pace of the whole kernel).
  if (warp == 0) {
    // ---------------- producer
    const bool leader = elect_one();
    const uint32_t full0 = CG == 2 ? in_cta(s_u32(full), 0) : s_u32(full);
    int s = 0, group = 0, mapped = -1;
    uint32_t round = 0;
    bool ok = true;
    for (int t = worker; t < tiles && ok; t += workers) {
      const Tile r = tile_at<CG, NT, MODE>(a, off, before, t, group);
      const int g = uniform(r.group), half = uniform(r.width) / CG;
      const int l = uniform(r.l0) + (int)half_rank * BM, c = uniform(r.c0) + (int)half_rank * half, k0 = uniform(r.k0), chunks = uniform(r.chunks);
      const CUtensorMap* ma = &tmA;
      // one box that covers this CTA's columns; rows of it past the tile's are not used
      const CUtensorMap* mb = half <= 32 ? &tmB32 : (half <= 64 ? &tmB64 : &tmB128);
      uint32_t b_bytes = (half <= 32 ? 32 : (half <= 64 ? 64 : 128)) * BK * 2;
      if (MODE == BACKWARD_WEIGHT) {
        ma = a.maps + 2 * g;
        mb = ma + 1;
        b_bytes = C::B_BYTES;
        if (mapped != g && chunks) {
          if (leader) {
            asm volatile("fence.proxy.tensormap::generic.acquire.gpu [%0], 128;" ::"l"(ma) : "memory");
            asm volatile("fence.proxy.tensormap::generic.acquire.gpu [%0], 128;" ::"l"(mb) : "memory");
          }
          mapped = g;
        }
      }
      const uint32_t bytes = CG * (A_BYTES + b_bytes);
      const int it1 = (part_rank + 1) * chunks / a.split;
      for (int it = part_rank * chunks / a.split; it < it1; ++it) {
        if (round && !__all_sync(0xffffffffu, wait(&empty[s], (round - 1) & 1u, abort_flag))) { ok = false; break; }
        unsigned char* sa = smem + s * C::STAGE;
        unsigned char* sb = sa + A_BYTES;
        const uint32_t bar = full0 + 8u * (uint32_t)s;
        const int k = k0 + it * BK;
        if (leader) {
          if (half_rank == 0) expect_tx(&full[s], bytes);
          if (MODE == FORWARD) {
            load_3d<CG>(sa, ma, k, l, g, bar);
          } else if (MODE == BACKWARD_DATA) {
            if (a.a_blocked) {
              load_4d<CG>(sa, ma, 0, k, l / 64, g, bar);
            } else {
              load_3d<CG>(sa, ma, l, k, g, bar);
              load_3d<CG>(sa + 8192, ma, l + 64, k, g, bar);
            }
          } else if (a.a_blocked) {
            load_3d<CG>(sa, ma, 0, k, l / 64, bar);
          } else {
            load_2d<CG>(sa, ma, l, k, bar);
            load_2d<CG>(sa + 8192, ma, l + 64, k, bar);
          }
          if (!B_MN) {
            load_2d<CG>(sb, mb, k, c, bar);
          } else if (a.b_blocked) {
            load_3d<CG>(sb, mb, 0, k, c / 64, bar);
          } else {
            load_2d<CG>(sb, mb, c, k, bar);
            load_2d<CG>(sb + 8192, mb, c + 64, k, bar);
          }
        }
        __syncwarp();
        if (++s == S) { s = 0; ++round; }
      }
    }
    if (*abort_flag)       // copies already issued land in a few microseconds; shared memory must outlive them
      for (int i = 0; i < 64; ++i) __nanosleep(20000);
  } else if (warp == 1 && half_rank == 0) {
    // ---------------- MMA issuer (of a pair: the even CTA)
    // K-major: 16 values are 32 bytes further along the swizzled row; 8-row groups 1024 bytes apart.  MN-major: 16
    // contraction rows are 2048 bytes further; 64-value blocks along the other dimension 8192 bytes apart.
    const bool leader = elect_one();
    const uint32_t sa0 = s_u32(smem), sb0 = sa0 + A_BYTES;
    const uint64_t a0 = A_MN ? smem_desc(sa0, 8192, 1024) : smem_desc(sa0, 16, 1024);
    const uint64_t b0 = B_MN ? smem_desc(sb0, 8192, 1024) : smem_desc(sb0, 16, 1024);
    constexpr uint32_t a_step = A_MN ? 2048 >> 4 : 32 >> 4, b_step = B_MN ? 2048 >> 4 : 32 >> 4;
    const uint32_t fixed = 1u << 4 | a.type_bits | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) | (uint32_t)(BM * CG / 16) << 24;
    const uint32_t tmem_u = (uint32_t)uniform((int)tmem_base);
    int s = 0, j = 0, group = 0;
    uint32_t round = 0, stage_off = 0;
    bool ok = true;
    for (int t = worker; t < tiles && ok; t += workers) {
      const Tile r = tile_at<CG, NT, MODE>(a, off, before, t, group);
      const int chunks = uniform(r.chunks);
      if (!chunks) continue;
      const int as = j & 1;
      if (j >= 2 && !__all_sync(0xffffffffu, wait(&acc_empty[as], (uint32_t)(((j >> 1) - 1) & 1), abort_flag))) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t acc = tmem_u + (uint32_t)(as * NT), idesc = fixed | (uint32_t)(uniform(r.width) >> 3) << 17;
      const int it0 = part_rank * chunks / a.split, it1 = (part_rank + 1) * chunks / a.split;
      for (int it = it0; it < it1; ++it) {
        if (!__all_sync(0xffffffffu, wait(&full[s], round & 1u, abort_flag))) { ok = false; break; }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint64_t da = a0 + stage_off, db = b0 + stage_off;
        const uint32_t done = s_u32(&empty[s]);
        if (leader) {
          mma<CG>(acc, da, db, idesc, it > it0 ? 1u : 0u);
#pragma unroll
          for (int kk = 1; kk < BK / 16; ++kk) mma<CG>(acc, da + kk * a_step, db + kk * b_step, idesc, 1u);
          commit<CG>(done);
        }
        __syncwarp();
        if (++s == S) { s = 0; ++round; stage_off = 0; } else stage_off += C::STAGE >> 4;
      }
      if (ok && leader) commit<CG>(s_u32(&acc_full[as]));
      __syncwarp();
      ++j;
    }
  } else if (warp >= 2) {
    // ---------------- epilogue: warp w reads accumulator lanes 32 * (w % 4) .. + 31, half of the columns
    const int q = warp & 3, part = (warp - 2) >> 2;
    int j = 0, group = 0;
    for (int t = worker; t < tiles; t += workers) {
      const Tile r = tile_at<CG, NT, MODE>(a, off, before, t, group);
      const int l = r.l0 + (int)half_rank * BM + q * 32 + lane;
      TO* out = (TO*)a.out + (MODE == BACKWARD_WEIGHT ? r.group * a.group_stride : 0) + (int64_t)r.c0 * a.ldo + l;
      const int chunks = (r.width + 31) / 32, c_begin = part ? (chunks + 1) / 2 : 0, c_end = part ? chunks : (chunks + 1) / 2;
      if (!r.chunks) {     // a group without rows: its gradient is zero
        if (l < a.lanes)
          for (int c = part; c < r.cols; c += 2) out[(int64_t)c * a.ldo] = from_f<TO>(0.f);
        continue;
      }
      const int as = j & 1;
      bool have = wait(&acc_full[as], (uint32_t)((j >> 1) & 1), abort_flag);
      have = __all_sync(0xffffffffu, have);
      if (!have) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      if (CG == 1 && a.split > 1) {      // this CTA's part of the sum to the first CTA, which stores the tile below
        mine = r; mine_l = l;
        if (part_rank > 0) {
          const uint32_t to = in_cta(s_u32(parts), 0) + (uint32_t)((part_rank - 1) * C::SPLIT_BYTES + (q * 32 + lane) * 4);
#pragma unroll 1
          for (int c = c_begin; c < c_end; ++c) {
            uint32_t v[32];
            tmem_load32(v, tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(c * 32));
#pragma unroll
            for (int k = 0; k < 32; ++k) asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(to + (c * 32 + k) * BM * 4), "r"(v[k]) : "memory");
          }
        }
        have_mine = true;
        break;
      }
#pragma unroll 1
      for (int c = c_begin; c < c_end; ++c) {
        if (c * 32 >= r.cols) break;
        uint32_t v[32];
        tmem_load32(v, tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(as * NT + c * 32));
        if (l < a.lanes) store_columns<TO>(out + (int64_t)(c * 32) * a.ldo, a.ldo, v, r.cols - c * 32);
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) {
        const uint32_t bar = CG == 2 ? in_cta(s_u32(&acc_empty[as]), 0) : s_u32(&acc_empty[as]);
        asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
      }
      ++j;
    }
    if (MODE != BACKWARD_WEIGHT) {       // rows beyond the last group: zeros
      for (int row = off[a.groups] + blockIdx.x * EPI_WARPS + warp - 2; row < a.rows; row += gridDim.x * EPI_WARPS)
        for (int l = lane; l < a.lanes; l += 32) ((TO*)a.out)[row * a.ldo + l] = from_f<TO>(0.f);
    }
  }
  __syncwarp();
  if (CG == 1 && a.split > 1) {
    cluster_sync_all();                  // the parts are in the first CTA's shared memory
    if (have_mine && part_rank == 0) {
      const int q = warp & 3, part = (warp - 2) >> 2, chunks = (mine.width + 31) / 32;
      TO* out = (TO*)a.out + (MODE == BACKWARD_WEIGHT ? mine.group * a.group_stride : 0) + (int64_t)mine.c0 * a.ldo + mine_l;
#pragma unroll 1
      for (int c = part ? (chunks + 1) / 2 : 0; c < (part ? chunks : (chunks + 1) / 2); ++c) {
        if (c * 32 >= mine.cols) break;
        uint32_t v[32];
        tmem_load32(v, tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(c * 32));
        const uint32_t from = s_u32(parts) + (uint32_t)((c * 32 * BM + q * 32 + lane) * 4);
        for (int p = 0; p + 1 < a.split; ++p) {          // in the parts' order
          float w[32];
#pragma unroll
          for (int k = 0; k < 32; ++k) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(w[k]) : "r"(from + (uint32_t)(p * C::SPLIT_BYTES + k * BM * 4)));
#pragma unroll
          for (int k = 0; k < 32; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) + w[k]);
        }
        if (mine_l < a.lanes) store_columns<TO>(out + (int64_t)(c * 32) * a.ldo, a.ldo, v, mine.cols - c * 32);
      }
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (CG == 2) cluster_sync_all();       // neither CTA leaves while the other may still signal its barriers
  if (*abort_flag && tid == 0) record_status(a.sb, BETTY_ERR_TIMEOUT);
  if (warp == 0) {
    if (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::TMEM_COLS) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::TMEM_COLS) : "memory");
  }
}

template <int NT, int MODE, typename TO>
__global__ void __launch_bounds__(THREADS, 1)
k_grouped(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB32, const __grid_constant__ CUtensorMap tmB64,
          const __grid_constant__ CUtensorMap tmB128, const Args a) {
  body<1, NT, MODE, TO>(tmA, tmB32, tmB64, tmB128, a);
}
template <int NT, int MODE, typename TO>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1)
k_grouped_pair(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB32, const __grid_constant__ CUtensorMap tmB64,
               const __grid_constant__ CUtensorMap tmB128, const Args a) {
  body<2, NT, MODE, TO>(tmA, tmB32, tmB64, tmB128, a);
}

// Writes group e's tensor maps of the weight gradient's operands: the given maps with the row extent cut at the group's end.
__global__ void __launch_bounds__(32)
k_group_maps(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const int32_t* offsets, int rows, CUtensorMap* maps) {
  __shared__ alignas(128) unsigned char buf[2][128];
  pdl_enter();
  const int e = blockIdx.x, lane = threadIdx.x;
  int end = 0;                                   // the clamped end of the group, as list_tiles takes it
  for (int i = lane; i <= e + 1; i += 32) end = max(end, min(offsets[i], rows));
  end = max(1, __reduce_max_sync(0xffffffffu, end));
  ((uint32_t*)buf[0])[lane] = ((const uint32_t*)&tmA)[lane];
  ((uint32_t*)buf[1])[lane] = ((const uint32_t*)&tmB)[lane];
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t s = s_u32(buf[i]);
    if (lane == 0)
      asm volatile("tensormap.replace.tile.global_dim.shared::cta.b1024.b32 [%0], 1, %1;" ::"r"(s), "r"(end) : "memory");
    __syncwarp();
    asm volatile("tensormap.cp_fenceproxy.global.shared::cta.tensormap::generic.release.gpu.sync.aligned [%0], [%1], 128;"
                 ::"l"(maps + 2 * e + i), "r"(s) : "memory");
  }
}

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

// ------------------------------------------------------------------ host side
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiledFn lookup_encode_fn() {
  void* p = nullptr;
  cudaDriverEntryPointQueryResult q;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess)
    return (EncodeTiledFn)p;
  (void)cudaGetLastError();
  return nullptr;
}
static EncodeTiledFn encode_fn() {
  static const EncodeTiledFn fn = lookup_encode_fn();
  return fn;
}

// an operand as the kernels read it: [groups][rows][cols], 16-bit values
struct Operand { const void* p; int64_t cols, rows, groups, ld, group_stride; };

static bool encode(CUtensorMap* tm, int dtype, int rank, const Operand& o, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  EncodeTiledFn fn = encode_fn();
  const cuuint32_t ones[4] = {1, 1, 1, 1};
  return fn && fn(tm, dtype == BETTY_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, (void*)o.p, dims, strides, box,
                  ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
static bool make_map(CUtensorMap* tm, int dtype, const Operand& o, bool three, int box_cols, int box_rows) {
  const cuuint64_t dims[3] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows, (cuuint64_t)o.groups};
  const cuuint64_t strides[2] = {(cuuint64_t)o.ld * 2, (cuuint64_t)o.group_stride * 2};
  const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1};
  return encode(tm, dtype, three ? 3 : 2, o, dims, strides, box);
}
// The same operand with its columns cut into blocks of 64 (their number a dimension of its own), so that one copy brings two
// blocks of 64 rows in the order that an MN-major operand wants: the issuing thread, not the bytes, bounds the loads
// otherwise.  Needs a multiple of 64 columns: a short last block would be read past its row.
static bool make_blocked_map(CUtensorMap* tm, int dtype, const Operand& o, bool three) {
  const cuuint64_t dims[4] = {64, (cuuint64_t)o.rows, (cuuint64_t)o.cols / 64, (cuuint64_t)o.groups};
  const cuuint64_t strides[3] = {(cuuint64_t)o.ld * 2, 128, (cuuint64_t)o.group_stride * 2};
  const cuuint32_t box[4] = {64, 64, 2, 1};
  return encode(tm, dtype, three ? 4 : 3, o, dims, strides, box);
}

static inline int64_t pad8(int64_t v) { return (v + 7) / 8 * 8; }

// The operand itself, or its rows copied to 16-byte boundaries in the workspace.
static betty_status align_operand(cudaStream_t stream, Arena& arena, Operand& o) {
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

template <int CG, int NT, int MODE, typename TO>
static betty_status launch_kernel(cudaStream_t stream, const CUtensorMap (&tm)[4], const Args& a, int64_t tiles) {
  const size_t smem = (size_t)Cfg<CG, NT>::smem(a.groups, a.split);
  static SmemLimit limit = {};
  auto kernel = [] {
    if constexpr (CG == 2) return k_grouped_pair<NT, MODE, TO>;
    else return k_grouped<NT, MODE, TO>;
  }();
  BETTY_TRY(ensure_dynamic_smem(kernel, limit, smem));
  const int64_t most = current_sm_count() / (CG * a.split);
  const int workers = (int)(tiles < 1 ? 1 : (tiles < most ? tiles : most));
  if (a.split == 1) {
    launch_pdl(kernel, dim3((unsigned)(workers * CG)), dim3(THREADS), smem, stream, tm[0], tm[1], tm[2], tm[3], a);
  } else {                 // as launch_pdl, with a cluster per tile
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(workers * a.split)); cfg.blockDim = dim3(THREADS); cfg.dynamicSmemBytes = smem; cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)a.split; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    (void)cudaLaunchKernelEx(&cfg, kernel, tm[0], tm[1], tm[2], tm[3], a);
  }
  BETTY_LAUNCH_CHECK();
  return BETTY_OK;
}

template <int CG, int NT, int MODE>
static betty_status run(cudaStream_t stream, Arena& arena, int dtype, int out_dtype, const Operand& A, const Operand& B, Args a) {
  CUtensorMap tm[4];
  bool ok;
  if (MODE == FORWARD) {
    ok = make_map(&tm[0], dtype, A, true, BK, BM);
  } else {
    a.a_blocked = A.cols % 64 == 0;
    ok = a.a_blocked ? make_blocked_map(&tm[0], dtype, A, MODE == BACKWARD_DATA) : make_map(&tm[0], dtype, A, MODE == BACKWARD_DATA, 64, BK);
  }
  if (MODE == BACKWARD_WEIGHT) {
    a.b_blocked = B.cols % 64 == 0;
    ok = ok && (a.b_blocked ? make_blocked_map(&tm[1], dtype, B, false) : make_map(&tm[1], dtype, B, false, 64, BK));
    tm[2] = tm[3] = tm[1];
  } else {
    ok = ok && make_map(&tm[1], dtype, B, false, BK, 32) && make_map(&tm[2], dtype, B, false, BK, 64) && make_map(&tm[3], dtype, B, false, BK, 128);
  }
  if (!ok) return BETTY_ERR_CUDA;
  const int64_t lane_tiles = (a.lanes + BM * CG - 1) / (BM * CG);
  int64_t tiles;           // an upper bound: the kernel knows the groups' rows, the host does not
  if (MODE == BACKWARD_WEIGHT) {
    CUtensorMap* maps = arena.alloc<CUtensorMap>(2 * (size_t)a.groups);
    if (!maps) return BETTY_ERR_WORKSPACE;
    a.maps = maps;
    launch_pdl(k_group_maps, dim3(a.groups), dim3(32), 0, stream, tm[0], tm[1], a.offsets, a.rows, maps);
    BETTY_LAUNCH_CHECK();
    tiles = lane_tiles * ((a.cols + NT - 1) / NT) * a.groups;
  } else {
    tiles = lane_tiles * (a.rows / NT + (a.rows < a.groups ? a.rows : a.groups));
    // few tiles: the CTAs of a cluster share each tile's contraction, eight chunks each or more
    const int chunks = (a.depth + BK - 1) / BK;
    if (CG == 1)
      while (a.split < Cfg<CG, NT>::MAX_SPLIT && tiles * a.split * 2 <= current_sm_count() && chunks >= 16 * a.split) a.split *= 2;
  }
  if (out_dtype == BETTY_F32) return launch_kernel<CG, NT, MODE, float>(stream, tm, a, tiles);
  if (dtype == BETTY_BF16) return launch_kernel<CG, NT, MODE, __nv_bfloat16>(stream, tm, a, tiles);
  return launch_kernel<CG, NT, MODE, __half>(stream, tm, a, tiles);
}

template <int MODE>
static betty_status product(const betty_grouped_cfg* c, int64_t rows, const int32_t* offsets, Operand A, Operand B, Args a, int out_dtype,
                            void* ws, size_t ws_bytes, void* stream) {
  const cudaStream_t s = (cudaStream_t)stream;
  Arena arena(ws, ws_bytes);
  a.offsets = offsets; a.groups = c->n_groups; a.rows = (int)rows; a.sb = arena.status();
  a.type_bits = c->dtype == BETTY_BF16 ? (1u << 7 | 1u << 10) : 0u;
  BETTY_TRY(align_operand(s, arena, A));
  BETTY_TRY(align_operand(s, arena, B));
  a.split = 1;
  if (MODE == BACKWARD_WEIGHT)
    return a.lanes > BM && a.cols > 128 ? run<2, 256, MODE>(s, arena, c->dtype, out_dtype, A, B, a) : run<1, 128, MODE>(s, arena, c->dtype, out_dtype, A, B, a);
  const int64_t used = rows < c->n_groups ? rows : c->n_groups, mean = (rows + used - 1) / used;
  const int64_t pair_tiles = (a.lanes + 2 * BM - 1) / (2 * BM) * ((mean + 255) / 256) * used;
  // Measured (bf16, us, launches in a row; pairs 256 wide / single SM 128 / 64 / 32): 24 rows, 8 experts, 1024 x 1024: 12.1 / 11.1 / 9.7 / 10.2; 1 row,
  // 4096 x 4096: 19.4 / 18.4 / 13.6 / 11.7 (the last two with split contractions); 200 rows, 8 experts, 4096 x 4096: 51.5 / 50.4 /
  // 50.3 / 61.7; 300 rows, 4 experts, 4096 -> 1024: 20.5 / 19.3 / 14.8 / 17.9; 800 rows, 4 experts, 1024 -> 2048: 11.7 / 9.3 /
  // 12.7 / 15.7; 5001 rows, 16 experts, 2048 -> 1024: 27.7 / 31.1 / 43.2 / 70.6.
  if (rows <= 32) return run<1, 32, MODE>(s, arena, c->dtype, out_dtype, A, B, a);
  if (mean <= 64 || (mean <= 128 && pair_tiles * 2 < current_sm_count() / 2)) return run<1, 64, MODE>(s, arena, c->dtype, out_dtype, A, B, a);
  if (a.lanes > BM && pair_tiles * 4 > current_sm_count()) return run<2, 256, MODE>(s, arena, c->dtype, out_dtype, A, B, a);
  return run<1, 128, MODE>(s, arena, c->dtype, out_dtype, A, B, a);
}

static betty_status check(const betty_grouped_cfg* c, int64_t rows, const int32_t* offsets, const void* ws, size_t ws_bytes) {
  if (!c || rows < 0) return BETTY_ERR_INVALID_ARG;
  if (c->dtype != BETTY_BF16 && c->dtype != BETTY_F16) return BETTY_ERR_DTYPE;
  if (c->n_groups < 1 || c->in < 1 || c->out < 1) return BETTY_ERR_SHAPE;
  // 32-bit tile counts and coordinates: at most 2^30 rows, 2^24 columns, 1024 groups
  if (c->n_groups > MAX_GROUPS || rows > (1 << 30) || c->in > (1 << 24) || c->out > (1 << 24)) return BETTY_ERR_UNSUPPORTED;
  if (((rows + 127) / 128 + c->n_groups) * ((c->out > c->in ? c->out : c->in) / 128 + 1) > (1 << 30) ||
      (int64_t)c->n_groups * (c->out / 128 + 1) * (c->in / 128 + 1) > (1 << 30))
    return BETTY_ERR_UNSUPPORTED;
  if (!offsets) return BETTY_ERR_INVALID_ARG;
  if ((uintptr_t)offsets & 3) return BETTY_ERR_ALIGNMENT;
  if (!ws || ws_bytes < sizeof(StatusBlock) || (((uintptr_t)ws) & 255u)) return BETTY_ERR_WORKSPACE;
  return BETTY_OK;
}
static betty_status check_matrix(const void* p, int64_t ld, int64_t rows, int64_t cols, int64_t bytes) {
  if (!p) return BETTY_ERR_INVALID_ARG;
  if (rows > 1 && ld < cols) return BETTY_ERR_SHAPE;
  return (uintptr_t)p % bytes ? BETTY_ERR_ALIGNMENT : BETTY_OK;
}
static betty_status check_groups(const betty_grouped_cfg* c, const void* p, int64_t ld, int64_t gs, int64_t bytes) {
  BETTY_TRY(check_matrix(p, ld, c->out, c->in, bytes));
  return c->n_groups > 1 && gs < (c->out - 1) * ld + c->in ? BETTY_ERR_SHAPE : BETTY_OK;
}
static betty_status out_size(const betty_grouped_cfg* c, int dtype, int64_t& bytes) {
  if (dtype != BETTY_F32 && dtype != c->dtype) return BETTY_ERR_DTYPE;
  bytes = dtype == BETTY_F32 ? 4 : 2;
  return BETTY_OK;
}

}  // namespace grouped
}  // namespace betty

using namespace betty;
using namespace betty::grouped;

extern "C" betty_status betty_grouped_workspace_size(const betty_grouped_cfg* cfg, int64_t rows, int32_t any_layout, size_t* bytes) {
  int32_t some = 0;
  if (!bytes) return BETTY_ERR_INVALID_ARG;
  BETTY_TRY(grouped::check(cfg, rows, &some, (const void*)256, 256));
  size_t n = sizeof(StatusBlock) + 256 + (size_t)cfg->n_groups * 2 * sizeof(CUtensorMap);
  if (any_layout) {
    const int64_t x = rows * pad8(cfg->in), y = rows * pad8(cfg->out), w = (int64_t)cfg->n_groups * cfg->out * pad8(cfg->in);
    const int64_t m = x < y ? x : y;               // two of the three are read by a call
    n += 2 * 256 + (size_t)(x + y + w - (m < w ? m : w)) * 2;
  }
  *bytes = n;
  return BETTY_OK;
}

extern "C" betty_status betty_grouped_forward(const betty_grouped_cfg* cfg, int64_t rows, const int32_t* offsets, const void* X, int64_t ldx,
                                              const void* W, int64_t ldw, int64_t group_stride, void* Y, int64_t ldy, int32_t y_dtype,
                                              void* ws, size_t ws_bytes, void* stream) {
  BETTY_TRY(grouped::check(cfg, rows, offsets, ws, ws_bytes));
  if (rows == 0) return BETTY_OK;
  int64_t yb;
  BETTY_TRY(out_size(cfg, y_dtype, yb));
  BETTY_TRY(grouped::check_matrix(X, ldx, rows, cfg->in, 2));
  BETTY_TRY(check_groups(cfg, W, ldw, group_stride, 2));
  BETTY_TRY(grouped::check_matrix(Y, ldy, rows, cfg->out, yb));
  grouped::Args a = {};
  a.lanes = (int)cfg->out; a.depth = (int)cfg->in; a.out = Y; a.ldo = ldy;
  const Operand A = {W, cfg->in, cfg->out, cfg->n_groups, ldw, group_stride}, B = {X, cfg->in, rows, 1, ldx, 0};
  return product<FORWARD>(cfg, rows, offsets, A, B, a, y_dtype, ws, ws_bytes, stream);
}

extern "C" betty_status betty_grouped_backward_data(const betty_grouped_cfg* cfg, int64_t rows, const int32_t* offsets, const void* dY,
                                                    int64_t lddy, const void* W, int64_t ldw, int64_t group_stride, void* dX, int64_t lddx,
                                                    int32_t dx_dtype, void* ws, size_t ws_bytes, void* stream) {
  BETTY_TRY(grouped::check(cfg, rows, offsets, ws, ws_bytes));
  if (rows == 0) return BETTY_OK;
  int64_t xb;
  BETTY_TRY(out_size(cfg, dx_dtype, xb));
  BETTY_TRY(grouped::check_matrix(dY, lddy, rows, cfg->out, 2));
  BETTY_TRY(check_groups(cfg, W, ldw, group_stride, 2));
  BETTY_TRY(grouped::check_matrix(dX, lddx, rows, cfg->in, xb));
  grouped::Args a = {};
  a.lanes = (int)cfg->in; a.depth = (int)cfg->out; a.out = dX; a.ldo = lddx;
  const Operand A = {W, cfg->in, cfg->out, cfg->n_groups, ldw, group_stride}, B = {dY, cfg->out, rows, 1, lddy, 0};
  return product<BACKWARD_DATA>(cfg, rows, offsets, A, B, a, dx_dtype, ws, ws_bytes, stream);
}

extern "C" betty_status betty_grouped_backward_weight(const betty_grouped_cfg* cfg, int64_t rows, const int32_t* offsets, const void* dY,
                                                      int64_t lddy, const void* X, int64_t ldx, void* dW, int64_t lddw, int64_t group_stride,
                                                      int32_t dw_dtype, void* ws, size_t ws_bytes, void* stream) {
  BETTY_TRY(grouped::check(cfg, rows, offsets, ws, ws_bytes));
  int64_t wb;
  BETTY_TRY(out_size(cfg, dw_dtype, wb));
  BETTY_TRY(check_groups(cfg, dW, lddw, group_stride, wb));
  if (rows > 0) {
    BETTY_TRY(grouped::check_matrix(dY, lddy, rows, cfg->out, 2));
    BETTY_TRY(grouped::check_matrix(X, ldx, rows, cfg->in, 2));
  }
  grouped::Args a = {};
  a.lanes = (int)cfg->in; a.cols = (int)cfg->out; a.out = dW; a.ldo = lddw; a.group_stride = group_stride;
  Operand A = {X, cfg->in, rows, 1, ldx, 0}, B = {dY, cfg->out, rows, 1, lddy, 0};
  if (rows == 0) {                               // the gradients are zero: maps that nothing is loaded through
    A.rows = B.rows = 1;
    A.p = B.p = ws;
  }
  return product<BACKWARD_WEIGHT>(cfg, rows, offsets, A, B, a, dw_dtype, ws, ws_bytes, stream);
}
