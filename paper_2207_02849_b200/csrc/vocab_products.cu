// The matrix products of the losses over a vocabulary: the logits, whose accumulators are turned into a row's statistics or
// into its gradient's coefficients before they leave the SM, and the two products of the gradients.
//
//   statistics   z = X W^T tile by tile; per row and half tile: max y, sum 2^(y - max), y at the row's entries
//   gradient     z again, dz = a 2^(y - lse2) + b - e p, rounded to the operands' type: a piece of the vocabulary at a time
//   products     dX += dz W over the piece's columns, dW = dz^T X over the rows; one launch for both
//
// An accumulator holds rows of the batch in its lanes and columns of the vocabulary, so a thread owns a row and its softmax
// statistics need no exchange.  Pairs of SMs take tiles of 256 x 256 (the widest instruction; each SM stages half of the operands, 64 KB
// for 8.4 MFLOP of a chunk), and two accumulators let a tile drain, in about 3 us, while the next is multiplied: with d of 700
// and more the products hide the epilogues.  A launch of the statistics, 8192 x 16384 x 4096: 656 us, 1.68 PFLOP/s; of the
// coefficients: 661 to 674; of both products: 1421 us, 1.55 PFLOP/s; the tensor pipe is 94 % busy in all.  With few rows (one tile
// of rows on single SMs) W's stream bounds all three: 24 x 32000 x 2048, 131 MB in 28 us; dX and dW 46 us (131 MB read again, 131
// written).
#include "vocab_loss.cuh"

namespace betty {
namespace vocab {
using namespace tc;

enum Mode { STATS = 0, GRAD = 1, PRODUCTS = 2 };

static constexpr int THREADS = 320;           // warp 0: TMA, warp 1: MMA, warps 2-9: epilogue
static constexpr int EPI_WARPS = 8;
static constexpr int STAGING = EPI_WARPS * 4096;   // each epilogue warp: 32 rows of 128 bytes, for its entries and its results

template <int CG, int NT> struct Cfg {
  static constexpr int STAGES = 192 * 1024;   // bytes of operands in flight
  static constexpr int MAX_STAGES = 16;
  static constexpr int SMEM = STAGES + STAGING + 512 + 1024;
  static constexpr int TMEM_COLS = 2 * NT;    // two accumulators: a tile drains while the next is multiplied
  static_assert(SMEM <= 227 * 1024 && MAX_STAGES * 16 + 48 <= 512, "shared memory");
};

struct alignas(64) Maps { CUtensorMap m[6]; };
// logits: operands by rows
enum { M_X = 0, M_W = 1, M_DZ_OUT = 2 };
// products: dz by rows and by blocks of columns, W and X by blocks of columns, the results
enum { M_DZ = 0, M_DZ_T = 1, M_W_T = 2, M_X_T = 3, M_DX = 4, M_DW = 5 };

struct Args {
  const Meta* meta;
  StatusBlock* sb;
  uint32_t type_bits;      // operand format bits of the instruction descriptor
  uint32_t a_bytes, b_bytes;   // bytes of the copies of A (by rows) and B of one CTA and chunk
  uint32_t stage;              // bytes of a stage: 128 rows of A, B
  int stages;
  int col0, cols;          // the piece of the vocabulary: first column, columns
  int d;
  int64_t rpad;
  // logits
  int width, band;         // columns of a tile; row tiles that are taken together
  int ahead;               // W may be asked for before the kernels before this one are done
  float c2;
  int top;
  const int2* entry;
  int rows;                // > 0: x is read in place, so many rows (statistics)
  const void* target; int id64; float share;
  float2* part; float* part_y; float* y_entry;
  const RowCoef* coef;
  uint16_t* dz; int64_t ldz;
  // products
  int twice;               // coefficients and products: remainders of the rounded coefficients, TWICE_ROWS rows behind them
  int want_dx, want_dw, add;          // add: dX's sums already hold the pieces before
  int w_blocked, dw_tma;
  void* dw; int64_t lddw;
};

// ------------------------------------------------------------------ tiles
struct Tile {
  int trans;               // A is dz^T
  int l0, c0;              // first lane (row, or column of the piece), first column (of the piece, or of d)
  int width;               // columns of the instruction
  int k0, chunks;          // contraction
  int part;                // split of dX's contraction, or column tile of the logits
};
struct Counts {
  int row_tiles, col_tiles, d_tiles, split;
  int first, second;       // tiles that are taken first (logits, dX), and then (dW)
  int lead;                // workers with one tile less of the first kind start this many tiles earlier with the second
};

template <int CG, int NT, int MODE>
__device__ __forceinline__ Counts count_tiles(const Args& a, int n, int split, int workers) {
  Counts c;
  c.split = split;
  c.second = c.lead = 0;
  if (MODE != PRODUCTS) {
    c.row_tiles = (n + BM * CG - 1) / (BM * CG);
    c.col_tiles = (a.cols + a.width - 1) / a.width;
    c.d_tiles = 0;
    c.first = c.row_tiles * c.col_tiles;
  } else {
    const Products p = products_of(n, a.d, a.cols, NT);
    c.row_tiles = p.row_tiles; c.col_tiles = p.col_tiles; c.d_tiles = p.d_tiles;
    c.first = a.want_dx ? p.row_tiles * p.d_tiles * split : 0;
    c.second = a.want_dw ? p.col_tiles * p.d_tiles : 0;
    if (c.first % workers) c.lead = (dx_cost(p, split) + dw_cost(p) / 2) / dw_cost(p);
  }
  return c;
}
// The i-th tile of a worker, -1 behind its last: the first kind in turn; then the second, which those whose turn it was not begin
// with `lead` tiles of, as long as a tile of the first kind takes, before all take turns again.
__device__ __forceinline__ int nth_tile(const Counts& c, int worker, int workers, int i) {
  const int rounds = c.first / workers, over = c.first - rounds * workers, mine = rounds + (worker < over);
  if (i < mine) return i * workers + worker;
  int j = i - mine;
  const int idle = workers - over;
  int t;
  if (worker >= over && j < c.lead) {
    t = j * idle + worker - over;
  } else {
    if (worker >= over) j -= c.lead;
    t = c.lead * idle + j * workers + worker;
  }
  return t < c.second ? c.first + t : -1;
}
// Tiles that run together are about as many along d as across it, so that they share what they read.
__device__ __forceinline__ void raster(int rows, int cols, int t, int& row, int& col) {
  constexpr int G = 8;
  const int per = rows * G, group = t / per, in = t - group * per, width = min(G, cols - group * G);
  row = in / width;
  col = group * G + in - row * width;
}
template <int CG, int NT, int MODE>
__device__ __forceinline__ Tile tile_at(const Args& a, const Counts& c, int n, int t) {
  Tile r;
  if (MODE != PRODUCTS) {
    const int per = a.band * c.col_tiles, band = t / per, in = t - band * per, height = min(a.band, c.row_tiles - band * a.band);
    r.trans = 0;
    r.part = in / height;
    r.l0 = (band * a.band + in - r.part * height) * (BM * CG);
    r.c0 = r.part * a.width;
    r.width = a.width;
    r.k0 = 0;
    r.chunks = (a.d + BK - 1) / BK;
  } else if (t < c.first) {
    int rest, dt;
    raster(c.row_tiles * c.split, c.d_tiles, t, rest, dt);
    const int chunks = (a.cols + BK - 1) / BK;
    r.trans = 0;
    r.c0 = dt * NT;
    r.width = a.d - r.c0 > NT / 2 ? NT : NT / 2;         // blocks of 64 columns in each CTA
    r.part = rest % c.split;
    r.l0 = rest / c.split * (BM * CG);
    const int k = (int)((int64_t)r.part * chunks / c.split);
    r.k0 = k * BK;
    r.chunks = (int)((int64_t)(r.part + 1) * chunks / c.split) - k;
  } else {
    t -= c.first;
    int rest, dt;
    raster(c.col_tiles, c.d_tiles, t, rest, dt);
    r.trans = 1;
    r.c0 = dt * NT;
    r.width = a.d - r.c0 > NT / 2 ? NT : NT / 2;
    r.part = 0;
    r.l0 = rest * (BM * CG);
    r.k0 = 0;
    r.chunks = (n + BK - 1) / BK;
  }
  return r;
}

// ------------------------------------------------------------------ epilogues
// A row's entries in ascending order of id, from the first at or behind a column; the next AHEAD of them are in registers, asked for
// together and before the accumulator is waited for, so that their latency is hidden behind the products.
struct Walk {
  static constexpr int AHEAD = 4;
  const int2* entry; int64_t stride;   // the row's first; from one to the next
  int at, end, left;       // place of q[0]; entries in q
  int2 q[AHEAD], then[AHEAD];
  __device__ __forceinline__ void ask(int from) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) then[i] = from + i < end ? entry[(from + i) * stride] : make_int2(NO_ID, 0);
  }
  __device__ __forceinline__ void fill() {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) q[i] = then[i];
    left = AHEAD;
    ask(at + AHEAD);
  }
  // the first entry at or behind the column: eight places are looked at at a time
  __device__ __forceinline__ void start(const int2* entries, int64_t apart, int top, int column) {
    entry = entries; stride = apart; end = top;
    int lo = 0, len = top > 1 ? top : 0;
    while (len > 0) {
      const int step = (len + 7) >> 3;
      int below = 0;
#pragma unroll
      for (int k = 1; k <= 8; ++k)
        if (k * step <= len) below += entry[(lo + k * step - 1) * stride].x < column;
      const int stop = lo + len;
      lo += below * step;
      len = min(step - 1, stop - lo);
    }
    at = lo;
    ask(at);
    fill();
    if (top == 1 && q[0].x < column) q[0].x = NO_ID;
  }
  __device__ __forceinline__ void none() {
    entry = nullptr; stride = 0; at = end = 0; left = AHEAD;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) q[i] = then[i] = make_int2(NO_ID, 0);
  }
  // a single entry
  __device__ __forceinline__ void one(int id, float share, int column) {
    none();
    if (id >= column) q[0] = make_int2(id, __float_as_int(share));
  }
  __device__ __forceinline__ int next() const { return q[0].x; }
  __device__ __forceinline__ float share() const { return __int_as_float(q[0].y); }
  __device__ __forceinline__ void step() {
    ++at;
    if (--left == 0) {
      fill();
    } else {
#pragma unroll
      for (int i = 0; i + 1 < AHEAD; ++i) q[i] = q[i + 1];
      q[AHEAD - 1].x = NO_ID;
    }
  }
};

template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *(const uint32_t*)&v;
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *(const uint32_t*)&v;
}

template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t v);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t v) { return __bfloat1622float2(*(const __nv_bfloat162*)&v); }
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t v) { return __half22float2(*(const __half2*)&v); }

__device__ __forceinline__ void store_2d(const CUtensorMap* tm, uint32_t from, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(tm), "r"(from), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void add_2d(const CUtensorMap* tm, uint32_t from, int x, int y) {
  asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.bulk_group [%0, {%2, %3}], [%1];" ::"l"(tm), "r"(from), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void prefetch_2d(const CUtensorMap* tm, int x, int y) {
  asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global [%0, {%1, %2}];" ::"l"(tm), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void to_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// 16 bytes of a row of 128 in the layout of a 128-byte swizzle
__device__ __forceinline__ void stage16(uint32_t rows, int row, int j, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(rows + (uint32_t)(row * 128 + ((j ^ (row & 7)) << 4))), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

// Registers have no index.  The entries among 32 columns go through the warp's staging, a lane's row each: the columns' values are put
// there for the entries to pick theirs, or the entries' shares for the columns to subtract.  A call of 10799 rows x 715 x 192 with 102
// entries a row takes 96 us; selecting them in registers, 31 or 64 instructions for the entries that the lanes have next, it took 132.
// Comparing an index with each of 32 registers by hand is no way out: the compiler makes an array in local memory of that, which is
// stored for every 32 columns, entries or not (8192 x 65536 x 4096: 3.27 ms, now 3.02).
__device__ __forceinline__ uint32_t staged_at(uint32_t rows, int row, int k) { return rows + (uint32_t)(row * 128 + (((k >> 2) ^ (row & 7)) << 4) + (k & 3) * 4); }
__device__ __forceinline__ float staged(uint32_t at) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}

// Columns [from, to) of a tile (its accumulator at `acc`, its first column of the vocabulary `c0`) to a row's statistics.
__device__ __forceinline__ void statistics(const Args& a, uint32_t acc, int c0, int from, int to, int limit, bool live, Walk& w, float* y_entry, float2* part,
                                           float* part_y, uint32_t mine) {
  const int lane = threadIdx.x & 31;
  float m = -INFINITY, s = 0.f, sum = 0.f;
#pragma unroll 1
  for (int c = from; c < to; c += 32) {
    uint32_t v[32];
    tmem_load32(v, acc + (uint32_t)c);
    const int cb = c0 + c, end = min(min(cb + 32, c0 + to), limit);     // columns that exist
    if (end < cb + 32) {
#pragma unroll
      for (int k = 0; k < 32; ++k)
        if (cb + k >= end) v[k] = __float_as_uint(-INFINITY);
    }
    float top[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) top[k] = __uint_as_float(v[k]);
#pragma unroll
    for (int k = 4; k < 32; ++k) top[k & 3] = fmaxf(top[k & 3], __uint_as_float(v[k]));
    const float most = fmaxf(m, fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * a.c2);
    const float base = most == -INFINITY ? 0.f : most;
    float e[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 32; ++k) e[k & 3] += exp2f(fmaf(__uint_as_float(v[k]), a.c2, -base));
    s = fmaf(s, exp2f(m - base), (e[0] + e[1]) + (e[2] + e[3]));
    m = most;
    if (part_y) {
      float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < 32; ++k) y[k & 3] += cb + k < end ? __uint_as_float(v[k]) : 0.f;
      sum += (y[0] + y[1]) + (y[2] + y[3]);
    }
    if (__any_sync(0xffffffffu, w.next() < end)) {
#pragma unroll
      for (int k = 0; k < 8; ++k) stage16(mine, lane, k, v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
      while (w.next() < end) {
        y_entry[w.at * a.rpad] = staged(staged_at(mine, lane, w.next() - cb)) * a.c2;
        w.step();
      }
      __syncwarp();
    }
  }
  if (live) {
    *part = make_float2(m, s);
    if (part_y) *part_y = sum * a.c2;
  }
}

// 32 columns of a tile as coefficients of a row's gradient, packed in pairs; rows that do not count and columns that do not exist: 0
// (rest: what the rounding took away, rounded itself; null: not wanted)
template <typename T>
__device__ __forceinline__ void coefficients(const Args& a, uint32_t acc, int cb, int end, bool live, const RowCoef& rc, Walk& w, uint32_t mine, uint32_t (&out)[16],
                                             uint32_t* rest = nullptr) {
  const int lane = threadIdx.x & 31;
  uint32_t v[32];
  tmem_load32(v, acc);
#pragma unroll
  for (int k = 0; k < 32; ++k) v[k] = __float_as_uint(fmaf(rc.a, exp2f(fmaf(__uint_as_float(v[k]), a.c2, -rc.lse2)), rc.b));
  if (__any_sync(0xffffffffu, w.next() < end)) {
    if (lane == 0) bulk_wait_read();             // of the results that were staged there before
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 8; ++k) stage16(mine, lane, k, 0u, 0u, 0u, 0u);
    while (w.next() < end) {
      const uint32_t at = staged_at(mine, lane, w.next() - cb);
      const float e = fmaf(rc.e, w.share(), staged(at));
      asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(e) : "memory");
      w.step();
    }
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      float e[4];
      asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(e[0]), "=f"(e[1]), "=f"(e[2]), "=f"(e[3]) : "r"(staged_at(mine, lane, 4 * k)) : "memory");
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * k + i] = __float_as_uint(__uint_as_float(v[4 * k + i]) - e[i]);
    }
    __syncwarp();
  }
  if (end < cb + 32 || !live) {
#pragma unroll
    for (int k = 0; k < 32; ++k)
      if (cb + k >= end || !live) v[k] = 0u;
  }
#pragma unroll
  for (int k = 0; k < 16; ++k) out[k] = pack2<T>(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1]));
  if (rest) {
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const float2 got = unpack2<T>(out[k]);
      rest[k] = pack2<T>(__uint_as_float(v[2 * k]) - got.x, __uint_as_float(v[2 * k + 1]) - got.y);
    }
  }
}

template <typename T> struct IsF32 { static constexpr bool value = false; };
template <> struct IsF32<float> { static constexpr bool value = true; };

// CG = 2: a pair of CTAs (a cluster of two) shares a tile of 256 lanes; each stages its own lanes of A and half of the
// columns of B, the even CTA issues the products, both hold the accumulator rows of their own lanes.
// T: the operands' type (logits' coefficients); TO: dW's type (products)
template <int CG, int NT, int MODE, typename T, typename TO>
__device__ __forceinline__ void body(const Maps& tm, const Args& a) {
  using C = Cfg<CG, NT>;
  const int S = a.stages;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  unsigned char* staging = smem + C::STAGES;
  uint64_t* full = (uint64_t*)(staging + STAGING);
  uint64_t* empty = full + C::MAX_STAGES;
  uint64_t* acc_full = empty + C::MAX_STAGES;
  uint64_t* acc_empty = acc_full + 2;
  uint32_t* tmem_slot = (uint32_t*)(acc_empty + 2);
  volatile int* abort_flag = (volatile int*)(tmem_slot + 1);

  const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
  uint32_t rank = 0;
  if (CG == 2) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const int worker = blockIdx.x / CG, workers = gridDim.x / CG;

  if (tid == 0) {
    for (int s = 0; s < S; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(&acc_full[s], 1); mbar_init(&acc_empty[s], CG * EPI_WARPS); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    for (int i = 0; i < (MODE == PRODUCTS ? 6 : 3); ++i) prefetch_map(&tm.m[i]);
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
  if (MODE != PRODUCTS && a.ahead && warp == 1 && elect_one()) {
    // a single row tile: which columns this CTA takes does not depend on the count of rows.  The first 512 KB are on the way to L2 while the
    // kernels before this one run (no read: what they still write to W, they write to L2 too)
    int left = (512 << 10) / (a.width / CG * BK * 2);
    for (int c = worker * a.width; c < a.cols; c += workers * a.width)
      for (int k = 0; k < a.d && left > 0; k += BK, --left) prefetch_2d(&tm.m[M_W], k, a.col0 + c + (int)rank * (a.width / CG));
  }
  pdl_enter();             // global memory is written, and read otherwise, from here on
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (CG == 2) cluster_sync_all();     // the other's barriers exist before anything is signalled across the cluster
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem_base = *tmem_slot;
  const int counted = MODE == STATS && a.rows ? a.rows : uniform(a.meta->n);
  const int n = MODE == PRODUCTS && a.twice && counted ? 2 * TWICE_ROWS : counted;
  const Counts count = count_tiles<CG, NT, MODE>(a, n, MODE == PRODUCTS ? uniform(a.meta->split) : 1, workers);

  // The loading and the multiplying warp run their loops with all lanes, and one lane issues (see grouped.cu).
  if (warp == 0) {
    // ---------------- producer
    const bool leader = elect_one();
    const uint32_t full0 = CG == 2 ? in_cta(s_u32(full), 0) : s_u32(full);
    int s = 0;
    uint32_t round = 0;
    bool ok = true;
    for (int i = 0; ok; ++i) {
      const int t = uniform(nth_tile(count, worker, workers, i));
      if (t < 0) break;
      const Tile r = tile_at<CG, NT, MODE>(a, count, n, t);
      const int trans = uniform(r.trans), chunks = uniform(r.chunks), k0 = uniform(r.k0);
      const int l = uniform(r.l0) + (int)rank * BM;
      const int c = (MODE == PRODUCTS ? 0 : a.col0) + uniform(r.c0) + (int)rank * (uniform(r.width) / CG);
      const uint32_t bytes = CG * ((trans ? (uint32_t)A_BYTES : a.a_bytes) + a.b_bytes);
      for (int it = 0; it < chunks; ++it) {
        if (round && !__all_sync(0xffffffffu, wait(&empty[s], (round - 1) & 1u, abort_flag))) { ok = false; break; }
        unsigned char* sa = smem + s * a.stage;
        unsigned char* sb = sa + A_BYTES;
        const uint32_t bar = full0 + 8u * (uint32_t)s;
        const int k = k0 + it * BK;
        if (leader) {
          if (rank == 0) expect_tx(&full[s], bytes);
          if (MODE != PRODUCTS) {
            load_2d<CG>(sa, &tm.m[M_X], k, l, bar);
            load_2d<CG>(sb, &tm.m[M_W], k, c, bar);
          } else if (trans) {
            load_3d<CG>(sa, &tm.m[M_DZ_T], 0, k, l / 64, bar);
            load_3d<CG>(sb, &tm.m[M_X_T], 0, k, c / 64, bar);
          } else {
            load_2d<CG>(sa, &tm.m[M_DZ], k, l, bar);
            if (a.w_blocked) {
              load_3d<CG>(sb, &tm.m[M_W_T], 0, a.col0 + k, c / 64, bar);
            } else {
              load_2d<CG>(sb, &tm.m[M_W_T], c, a.col0 + k, bar);
              load_2d<CG>(sb + 8192, &tm.m[M_W_T], c + 64, a.col0 + k, bar);
            }
          }
        }
        __syncwarp();
        if (++s == S) { s = 0; ++round; }
      }
    }
    if (*abort_flag)       // copies already issued land in a few microseconds; shared memory must outlive them
      for (int i = 0; i < 64; ++i) __nanosleep(20000);
  } else if (warp == 1 && rank == 0) {
    // ---------------- MMA issuer (of a pair: the even CTA)
    // K-major: 16 values are 32 bytes further along the swizzled row; 8-row groups 1024 bytes apart.  MN-major: 16
    // contraction rows are 2048 bytes further; 64-value blocks along the other dimension 8192 bytes apart.
    const bool leader = elect_one();
    const uint32_t sa0 = s_u32(smem), sb0 = sa0 + A_BYTES;
    const uint64_t a_rows = smem_desc(sa0, 16, 1024), a_cols = smem_desc(sa0, 8192, 1024);
    const uint64_t b0 = MODE == PRODUCTS ? smem_desc(sb0, 8192, 1024) : smem_desc(sb0, 16, 1024);
    constexpr uint32_t b_step = MODE == PRODUCTS ? 2048 >> 4 : 32 >> 4;
    const uint32_t fixed = 1u << 4 | a.type_bits | (MODE == PRODUCTS ? 1u << 16 : 0u) | (uint32_t)(BM * CG / 16) << 24;
    const uint32_t tmem_u = (uint32_t)uniform((int)tmem_base);
    int s = 0, j = 0;
    uint32_t round = 0, stage_off = 0;
    bool ok = true;
    for (int i = 0; ok; ++i) {
      const int t = uniform(nth_tile(count, worker, workers, i));
      if (t < 0) break;
      const Tile r = tile_at<CG, NT, MODE>(a, count, n, t);
      const int chunks = uniform(r.chunks), trans = uniform(r.trans);
      if (!chunks) continue;
      const int as = j & 1;
      if (j >= 2 && !__all_sync(0xffffffffu, wait(&acc_empty[as], (uint32_t)(((j >> 1) - 1) & 1), abort_flag))) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t acc = tmem_u + (uint32_t)(as * NT), idesc = fixed | (uint32_t)trans << 15 | (uint32_t)(uniform(r.width) >> 3) << 17;
      const uint64_t a0 = trans ? a_cols : a_rows;
      const uint32_t a_step = trans ? 2048 >> 4 : 32 >> 4;
      // a contraction over the rows ends with the 16 that hold the last of them: what the copies behind those hold is not looked at
      const int last = trans ? (n + 15) / 16 - (chunks - 1) * (BK / 16) : BK / 16;
      for (int it = 0; it < chunks; ++it) {
        if (!__all_sync(0xffffffffu, wait(&full[s], round & 1u, abort_flag))) { ok = false; break; }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint64_t da = a0 + stage_off, db = b0 + stage_off;
        const uint32_t done = s_u32(&empty[s]);
        if (leader) {
          mma<CG>(acc, da, db, idesc, it ? 1u : 0u);
#pragma unroll
          for (int kk = 1; kk < BK / 16; ++kk)
            if (kk < last || it + 1 < chunks) mma<CG>(acc, da + kk * a_step, db + kk * b_step, idesc, 1u);
          commit<CG>(done);
        }
        __syncwarp();
        if (++s == S) { s = 0; ++round; stage_off = 0; } else stage_off += a.stage >> 4;
      }
      if (ok && leader) commit<CG>(s_u32(&acc_full[as]));
      __syncwarp();
      ++j;
    }
  } else if (warp >= 2) {
    // ---------------- epilogue: warp w reads accumulator lanes 32 * (w % 4) .. + 31, half of the columns
    const int q = warp & 3, part = (warp - 2) >> 2;
    const uint32_t mine = s_u32(staging) + (uint32_t)(warp - 2) * 4096u;
    const float dw_scale = MODE == PRODUCTS ? a.meta->dw_scale : 1.f;
    const int padded = MODE == GRAD && a.twice ? TWICE_ROWS : (n + 15) / 16 * 16;   // rows of dz that a contraction over the rows takes
    int j = 0;
    const int split_rows = count.row_tiles * (BM * CG);  // rows of one part of dX's sums
    for (int i = 0;; ++i) {
      const int t = nth_tile(count, worker, workers, i);
      if (t < 0) break;
      const Tile r = tile_at<CG, NT, MODE>(a, count, n, t);
      const int as = j & 1;
      const int first = r.l0 + (int)rank * BM + q * 32, row = first + lane;
      // logits: this warp's columns of the tile; the row's entries there and its coefficients, before the accumulator is waited for
      const int half = MODE == PRODUCTS ? NT / 2 : ((a.width + 63) >> 6) << 5, from = part ? half : 0, to = MODE == PRODUCTS || !part ? half : a.width;
      const bool live = row < n;
      Walk w;
      RowCoef rc = {0.f, 0.f, 0.f, 0.f};
      if (MODE != PRODUCTS) {
        w.none();
        if (live) {
          if (MODE == GRAD) rc = a.coef[row];
          if (MODE == STATS && a.target) {
            const int64_t id = a.id64 ? ((const int64_t*)a.target)[row] : ((const int32_t*)a.target)[row];
            w.one(id >= 0 && id < a.cols ? (int)id : -1, a.share, r.c0 + from);
          } else {
            w.start(a.entry + row, a.rpad, a.top, a.col0 + r.c0 + from);
          }
        }
      }
      if (r.chunks) {
        bool have = wait(&acc_full[as], (uint32_t)((j >> 1) & 1), abort_flag);
        have = __all_sync(0xffffffffu, have);
        if (!have) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      }
      const uint32_t acc = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(as * NT);
      if (MODE == STATS) {
        if (first < n) {
          const int64_t at = (int64_t)(r.part * 2 + part) * a.rpad + row;
          statistics(a, acc, r.c0, from, to, a.cols, live, w, a.y_entry + row, a.part + at, a.part_y ? a.part_y + at : nullptr, mine);
        }
      } else if (MODE == GRAD) {
        if (first < padded) {
          const int limit = min(a.cols, r.c0 + a.width), shift = a.col0;
          if (CG == 2) {
#pragma unroll 1
            for (int c = from; c < to; c += 64) {
              const int x = r.c0 + c;
              if (x >= a.cols) break;
              uint32_t lo[16], hi[16];
              coefficients<T>(a, acc + (uint32_t)c, shift + x, shift + min(x + 32, limit), live, rc, w, mine, lo);
              coefficients<T>(a, acc + (uint32_t)(c + 32), shift + x + 32, shift + max(x + 32, min(x + 64, limit)), live, rc, w, mine, hi);
              if (lane == 0) bulk_wait_read();
              __syncwarp();
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                stage16(mine, lane, k, lo[4 * k], lo[4 * k + 1], lo[4 * k + 2], lo[4 * k + 3]);
                stage16(mine, lane, 4 + k, hi[4 * k], hi[4 * k + 1], hi[4 * k + 2], hi[4 * k + 3]);
              }
              to_async_proxy();
              __syncwarp();
              if (lane == 0) { store_2d(&tm.m[M_DZ_OUT], mine, x, first); bulk_commit(); }
            }
          } else {
            uint16_t* out = a.dz + (int64_t)row * a.ldz + r.c0;
#pragma unroll 1
            for (int c = from; c < to; c += 32) {
              const int x = r.c0 + c;
              if (x >= a.cols) break;
              uint32_t v[16], rest[16];
              const int end = shift + min(min(x + 32, r.c0 + to), limit);
              coefficients<T>(a, acc + (uint32_t)c, shift + x, end, live, rc, w, mine, v, a.twice ? rest : nullptr);
              if (row < padded) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  if (c + 8 * k >= to || x + 8 * k >= a.cols) break;
                  *(uint4*)(out + c + 8 * k) = make_uint4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
                  if (a.twice) *(uint4*)(out + TWICE_ROWS * a.ldz + c + 8 * k) = make_uint4(rest[4 * k], rest[4 * k + 1], rest[4 * k + 2], rest[4 * k + 3]);
                }
              }
            }
          }
        }
      } else {
        const int x0 = r.c0 + part * (NT / 2);
        if (!r.trans || IsF32<TO>::value) {
          const float f = r.trans ? dw_scale : 1.f;
          const bool wanted = r.trans ? first < a.cols : first < n && r.chunks;   // the last piece may be shorter than its parts are many
          if (wanted) {
#pragma unroll 1
            for (int c = 0; c < NT / 2; c += 32) {
              if (x0 + c >= a.d) break;
              uint32_t v[32];
              if (r.chunks) tmem_load32(v, acc + (uint32_t)(part * (NT / 2) + c));
              if (lane == 0) bulk_wait_read();
              __syncwarp();
              if (r.trans) {
#pragma unroll
                for (int k = 0; k < 32; ++k) v[k] = r.chunks ? __float_as_uint(__uint_as_float(v[k]) * f) : 0u;
              }
#pragma unroll
              for (int k = 0; k < 8; ++k) stage16(mine, lane, k, v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
              if (!r.trans || a.dw_tma) {
                to_async_proxy();
                __syncwarp();
                if (lane == 0) {
                  if (r.trans) store_2d(&tm.m[M_DW], mine, x0 + c, a.col0 + first);
                  else if (a.add) add_2d(&tm.m[M_DX], mine, x0 + c, r.part * split_rows + first);
                  else store_2d(&tm.m[M_DX], mine, x0 + c, r.part * split_rows + first);
                  bulk_commit();
                }
              } else {       // rows of dW that do not start on 16-byte boundaries
                __syncwarp();
                float* out = (float*)a.dw + (int64_t)(a.col0 + first) * a.lddw + x0 + c;
                for (int i = 0; i < 32 && first + i < a.cols; ++i) {
                  uint32_t u;
                  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(u) : "r"(mine + (uint32_t)(i * 128 + (((lane >> 2) ^ (i & 7)) << 4) + (lane & 3) * 4)) : "memory");
                  if (x0 + c + lane < a.d) out[(int64_t)i * a.lddw + lane] = __uint_as_float(u);
                }
                __syncwarp();
              }
            }
          }
        } else if (first < a.cols) {
          if constexpr (!IsF32<TO>::value) {
#pragma unroll 1
            for (int c = 0; c < NT / 2; c += 64) {
              if (x0 + c >= a.d) break;
              if (lane == 0) bulk_wait_read();
              __syncwarp();
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                uint32_t v[32];
                if (r.chunks) {
                  tmem_load32(v, acc + (uint32_t)(part * (NT / 2) + c + h * 32));
                } else {
#pragma unroll
                  for (int k = 0; k < 32; ++k) v[k] = 0u;
                }
                uint32_t u[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) u[k] = pack2<TO>(__uint_as_float(v[2 * k]) * dw_scale, __uint_as_float(v[2 * k + 1]) * dw_scale);
#pragma unroll
                for (int k = 0; k < 4; ++k) stage16(mine, lane, h * 4 + k, u[4 * k], u[4 * k + 1], u[4 * k + 2], u[4 * k + 3]);
              }
              if (a.dw_tma) {
                to_async_proxy();
                __syncwarp();
                if (lane == 0) { store_2d(&tm.m[M_DW], mine, x0 + c, a.col0 + first); bulk_commit(); }
              } else {
                __syncwarp();
                uint16_t* out = (uint16_t*)a.dw + (int64_t)(a.col0 + first) * a.lddw + x0 + c;
                for (int i = 0; i < 32 && first + i < a.cols; ++i) {
#pragma unroll
                  for (int h = 0; h < 2; ++h) {
                    const int e = h * 32 + lane;
                    uint16_t u;
                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(u) : "r"(mine + (uint32_t)(i * 128 + (((e >> 3) ^ (i & 7)) << 4) + (e & 7) * 2)) : "memory");
                    if (x0 + c + e < a.d) out[(int64_t)i * a.lddw + e] = u;
                  }
                }
                __syncwarp();
              }
            }
          }
        }
      }
      if (r.chunks) {
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          const uint32_t bar = CG == 2 ? in_cta(s_u32(&acc_empty[as]), 0) : s_u32(&acc_empty[as]);
          asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
        }
        ++j;
      }
    }
    if (lane == 0) bulk_wait_all();
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (CG == 2) cluster_sync_all();       // neither CTA leaves while the other may still signal its barriers
  if (*abort_flag && tid == 0) record_status(a.sb, BETTY_ERR_TIMEOUT);
  if (warp == 0) {
    if (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::TMEM_COLS) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::TMEM_COLS) : "memory");
  }
}

template <int NT, int MODE, typename T, typename TO>
__global__ void __launch_bounds__(THREADS, 1) k_vocab(const __grid_constant__ Maps tm, const Args a) {
  body<1, NT, MODE, T, TO>(tm, a);
}
template <int NT, int MODE, typename T, typename TO>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1) k_vocab_pair(const __grid_constant__ Maps tm, const Args a) {
  body<2, NT, MODE, T, TO>(tm, a);
}

// ------------------------------------------------------------------ host side
template <int CG, int NT, int MODE, typename T, typename TO>
static betty_status launch(cudaStream_t stream, const Maps& tm, const Args& a, int64_t tiles) {
  static SmemLimit limit = {};
  auto kernel = [] {
    if constexpr (CG == 2) return k_vocab_pair<NT, MODE, T, TO>;
    else return k_vocab<NT, MODE, T, TO>;
  }();
  BETTY_TRY(ensure_dynamic_smem(kernel, limit, (size_t)Cfg<CG, NT>::SMEM));
  const int64_t most = current_sm_count() / CG;
  const int workers = (int)(tiles < 1 ? 1 : (tiles < most ? tiles : most));
  launch_pdl(kernel, dim3((unsigned)(workers * CG)), dim3(THREADS), (size_t)Cfg<CG, NT>::SMEM, stream, tm, a);
  BETTY_LAUNCH_CHECK();
  return BETTY_OK;
}

static int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// A matrix by rows: boxes of `box_cols` values of `box_rows` rows
static bool map_rows(CUtensorMap* tm, CUtensorMapDataType type, int bytes, const void* p, int64_t cols, int64_t rows, int64_t ld, int box_cols, int box_rows) {
  EncodeTiledFn fn = encode_fn();
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * bytes};
  const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, ones[2] = {1, 1};
  return fn && fn(tm, type, 2, (void*)p, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static int box_rows_of(int rows) { return rows <= 32 ? 32 : (rows <= 64 ? 64 : 128); }

// A stage has room for all 128 rows of A: of few rows only those are copied, the others hold what was there before and end in accumulator
// lanes that nothing looks at.  (Room for the copied rows alone, and more stages for it, was no faster: 8 rows 21.8 us, with whole
// ones 22.3; 24 rows, gradients, 91.1 and 87.8.)
static void set_stages(Args& a) {
  a.stage = A_BYTES + a.b_bytes;
  const int fit = Cfg<1, 128>::STAGES / (int)a.stage;
  a.stages = fit < Cfg<1, 128>::MAX_STAGES ? fit : Cfg<1, 128>::MAX_STAGES;
}

int logits_parts(const Shape& s) { return 2 * (int)div_up(s.vocab, s.width); }

static void common_args(Args& a, const Shape& s, const Buffers& b) {
  a.meta = b.meta; a.sb = b.sb;
  a.type_bits = s.dtype == BETTY_BF16 ? (1u << 7 | 1u << 10) : 0u;
  a.d = s.d; a.rpad = s.rpad;
  a.width = s.width; a.c2 = s.c2; a.top = s.top;
  a.entry = b.entry;
  // the row tiles whose copies of x are taken together stay in L2 while W streams past them: 32 MB of it
  const int64_t tile_bytes = (s.pairs ? 256 : 128) * s.dp * 2;
  a.band = (int)(tile_bytes >= (32 << 20) ? 1 : (32 << 20) / tile_bytes);
}
static betty_status logits_maps(Maps& tm, Args& a, const Shape& s, const Buffers& b, const Operand& w) {
  const CUtensorMapDataType type = s.dtype == BETTY_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  const int a_box = s.pairs ? 128 : box_rows_of(s.rows), b_box = s.pairs ? 128 : s.width;
  a.a_bytes = (uint32_t)a_box * BK * 2; a.b_bytes = (uint32_t)b_box * BK * 2;
  set_stages(a);
  if (!map_rows(&tm.m[M_X], type, 2, b.x, s.dp, s.rpad, s.dp, BK, a_box)) return BETTY_ERR_CUDA;
  if (!map_rows(&tm.m[M_W], type, 2, w.p, w.cols, w.rows, w.ld, BK, b_box)) return BETTY_ERR_CUDA;
  tm.m[M_DZ_OUT] = tm.m[M_X];
  return BETTY_OK;
}

betty_status logits_statistics(cudaStream_t stream, const Shape& s, const Buffers& b, const Operand& w, bool w_ahead, const InPlace* in_place) {
  Maps tm;
  Args a = {};
  common_args(a, s, b);
  a.cols = s.vocab;
  a.part = b.part; a.part_y = b.part_y; a.y_entry = b.y_entry;
  BETTY_TRY(logits_maps(tm, a, s, b, w));
  a.ahead = w_ahead && s.rows <= 128;
  if (in_place) {
    a.rows = s.rows; a.target = in_place->target; a.id64 = in_place->id64; a.share = in_place->share;
    const CUtensorMapDataType type = s.dtype == BETTY_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    if (!map_rows(&tm.m[M_X], type, 2, in_place->x, s.d, s.rows, in_place->ldx, BK, box_rows_of(s.rows))) return BETTY_ERR_CUDA;
  }
  const int64_t tiles = div_up(s.rows, s.pairs ? 256 : 128) * div_up(s.vocab, s.width);
  // the operands' type is in the instruction descriptor: nothing else of the statistics depends on it
  if (s.pairs) return launch<2, 256, STATS, __nv_bfloat16, float>(stream, tm, a, tiles);
  return launch<1, 256, STATS, __nv_bfloat16, float>(stream, tm, a, tiles);
}

template <typename T>
static betty_status launch_grad(cudaStream_t stream, const Shape& s, const Maps& tm, const Args& a) {
  const int64_t tiles = div_up(s.rows, s.pairs ? 256 : 128) * div_up(a.cols, s.width);
  if (s.pairs) return launch<2, 256, GRAD, T, float>(stream, tm, a, tiles);
  return launch<1, 256, GRAD, T, float>(stream, tm, a, tiles);
}
template <typename TO>
static betty_status launch_products(cudaStream_t stream, const Shape& s, const Maps& tm, const Args& a) {
  const int lanes = s.product_pairs ? 256 : 128, nt = lanes;
  const int64_t tiles = ((a.want_dx ? s.sum_rows / lanes : 0) + (a.want_dw ? div_up(a.cols, lanes) : 0)) * div_up(s.d, nt);
  if (s.product_pairs) return launch<2, 256, PRODUCTS, __nv_bfloat16, TO>(stream, tm, a, tiles);
  return launch<1, 128, PRODUCTS, __nv_bfloat16, TO>(stream, tm, a, tiles);
}

betty_status logits_gradients(cudaStream_t stream, const Shape& s, const Buffers& b, const Operand& w, bool w_ahead, void* dw, int64_t lddw, int dw_dtype) {
  const CUtensorMapDataType type = s.dtype == BETTY_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  Maps lm, pm;
  Args la = {}, pa = {};
  common_args(la, s, b);
  BETTY_TRY(logits_maps(lm, la, s, b, w));
  la.coef = b.coef; la.dz = b.dz; la.ldz = s.piece;
  if (s.pairs && !map_rows(&lm.m[M_DZ_OUT], type, 2, b.dz, s.piece, s.rpad, s.piece, 64, 32)) return BETTY_ERR_CUDA;

  common_args(pa, s, b);
  pa.want_dx = s.want_dx; pa.want_dw = s.want_dw;
  pa.w_blocked = w.cols % 64 == 0;
  pa.dw = dw; pa.lddw = lddw;
  const int a_box = s.product_pairs ? 128 : box_rows_of(s.twice ? 2 * TWICE_ROWS : s.rows);
  la.twice = pa.twice = s.twice;
  pa.a_bytes = (uint32_t)a_box * BK * 2; pa.b_bytes = 128 * BK * 2;
  set_stages(pa);
  const Operand dz = {b.dz, s.piece, s.rpad, 1, s.piece, 0}, x = {b.x_dw, s.dp, s.rpad, 1, s.dp, 0};
  bool ok = make_blocked_map(&pm.m[M_DZ_T], s.dtype, dz, false) && make_blocked_map(&pm.m[M_X_T], s.dtype, x, false);
  ok = ok && (pa.w_blocked ? make_blocked_map(&pm.m[M_W_T], s.dtype, w, false) : make_map(&pm.m[M_W_T], s.dtype, w, false, 64, BK));
  pm.m[M_DX] = pm.m[M_DW] = pm.m[M_DZ_T];
  if (s.want_dx) ok = ok && map_rows(&pm.m[M_DX], CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, b.dx, s.dp, s.sum_rows, s.dp, 32, 32);
  const int ob = dw_dtype == BETTY_F32 ? 4 : 2;
  if (s.vocab == 1) lddw = pad8(s.d);            // a stride that is never used still has to be a valid one
  // a TMA store writes whole 16-byte pieces: where a row does not end with one, what lies behind it would be overwritten
  if (dw && aligned16(dw) && (lddw * ob) % 16 == 0 && ((int64_t)s.d * ob) % 16 == 0) {
    pa.dw_tma = 1;
    ok = ok && map_rows(&pm.m[M_DW], dw_dtype == BETTY_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : type, ob, dw, s.d, s.vocab, lddw, 128 / ob, 32);
  }
  if (!ok) return BETTY_ERR_CUDA;

  for (int c = 0; c < s.vocab; c += s.piece) {
    la.col0 = pa.col0 = c;
    la.cols = pa.cols = s.vocab - c < s.piece ? s.vocab - c : s.piece;
    pa.add = c > 0;
    la.ahead = w_ahead && s.rows <= 128 && c == 0;
    // columns behind the vocabulary's last are not in the map: the contraction reads zeros there
    if ((c == 0 || pa.cols < s.piece) && !map_rows(&pm.m[M_DZ], type, 2, b.dz, pa.cols, s.rpad, s.piece, BK, a_box)) return BETTY_ERR_CUDA;
    BETTY_TRY(s.dtype == BETTY_BF16 ? launch_grad<__nv_bfloat16>(stream, s, lm, la) : launch_grad<__half>(stream, s, lm, la));
    BETTY_TRY(dw_dtype == BETTY_F32 ? launch_products<float>(stream, s, pm, pa)
                                    : (s.dtype == BETTY_BF16 ? launch_products<__nv_bfloat16>(stream, s, pm, pa) : launch_products<__half>(stream, s, pm, pa)));
  }
  return BETTY_OK;
}

// Which tiles, and how much of the vocabulary at a time.
void choose_shape(Shape& s, bool backward) {
  const int64_t sms = current_sm_count(), rows = s.rows < 1 ? 1 : s.rows;
  s.piece = (int)(div_up(s.vocab, 256) * 256);
  if (backward) {
    // coefficients of 256 MB: fewer, longer pieces have fewer ends and fewer additions to dX's sums (8192 x 65536 x 4096 in 16 / 8 / 4
    // pieces: 9.38 / 9.17 / 9.27 ms; 1640 of 4096 rows x 32000 x 2048 in 4 / 2 / 1: 535 / 500 / 488 us)
    const int64_t most = (int64_t)1 << 27, fits = most / s.rpad / 256 * 256, piece = fits < 1024 ? 1024 : fits;
    const int64_t pieces = div_up(s.vocab, piece);
    s.piece = (int)(div_up(div_up(s.vocab, pieces), 256) * 256);
  }
  const int64_t cols = backward ? (s.piece < s.vocab ? s.piece : s.vocab) : s.vocab;
  // Tiles of the logits: pairs take 256 x 256, a single SM 128 rows x width.  Time of the rounds in us: a contraction chunk takes 0.34 in
  // a pair; alone 0.27 for any width up to 112 and little more above with one tile of rows, but 0.53 for 256 columns with several
  // (777 rows x 12345 x 1537: 44.7 us, pairs 27.9), and a tile is drained while the next is multiplied, 256 columns in 3 us in a
  // pair, alone somewhat slower (1293 rows x 116984 x 128, gradients: 279 us, pairs 225).
  const double chunks = (double)div_up(s.d, BK);
  double best = 1e30;
  for (int w = 32; w <= 272; w += 16) {
    const bool pair = w > 256;
    if (pair && rows <= 128) break;
    const int64_t rounds = pair ? div_up(div_up(rows, 256) * div_up(cols, 256), sms / 2) : div_up(div_up(rows, 128) * div_up(cols, w), sms);
    const double multiply = chunks * (pair ? 0.34 : 0.25 + (rows <= 128 ? 0.09 : 0.28) * w / 256), drain = pair ? 3.0 : 0.4 + (backward ? 4.4 : 3.0) * w / 256;
    const double time = (double)rounds * (multiply > drain ? multiply : drain) + (multiply > drain ? drain : multiply);
    if (time <= best) { best = time; s.pairs = pair; s.width = pair ? 256 : w; }
  }
  s.product_pairs = 0;
  s.sum_rows = s.rpad;
  s.twice = backward && rows <= TWICE_ROWS;
  if (!backward) return;
  const int64_t pair_tiles = div_up(s.d, 256) * ((s.want_dx ? div_up(rows, 256) : 0) + (s.want_dw ? div_up(s.piece, 256) : 0));
  s.product_pairs = rows > 128 && pair_tiles * 2 >= sms / 2;
  // dX with few rows: room for parts of its contraction, of 8 chunks or more, that are up to two tiles for each worker, and 32 at most
  // (8 rows x 56960 x 64 in 111 parts: 20 us to add them up, in 32: 6); k_rows chooses their number once the rows are counted
  const int lanes = s.product_pairs ? 256 : 128;
  const int64_t tiles = div_up(rows, lanes) * div_up(s.d, lanes), workers = s.product_pairs ? sms / 2 : sms;
  int64_t parts = div_up(2 * workers, tiles);
  if (parts > div_up(cols, BK) / 8) parts = div_up(cols, BK) / 8;
  s.sum_rows = s.rpad * (parts < 1 ? 1 : (parts < 32 ? parts : 32));
}

}  // namespace vocab
}  // namespace betty
