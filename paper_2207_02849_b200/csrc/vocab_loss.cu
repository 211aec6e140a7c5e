// Losses over a vocabulary: the rows that count and their entries, the losses from the statistics of the logits' tiles, and the
// C entries (see vocab_loss.cuh for the mathematics).
//
// What surrounds the products is bound by memory and small beside them, with few rows by latency: a copy of x in (8192 x 4096: 134 MB in 22
// to 26 us), 8 bytes of statistics per row and half tile (8192 rows of 128 parts: 7 us), fp32 sums of dX out (201 MB in 45 to 50 us).
#include "vocab_loss.cuh"

namespace betty {
namespace vocab {
using namespace tc;

static constexpr int ROW_THREADS = 256;

// ------------------------------------------------------------------ values of the caller's types
__device__ __forceinline__ int64_t whole(const void* p, int is64, int64_t i) { return is64 ? ((const int64_t*)p)[i] : ((const int32_t*)p)[i]; }
__device__ __forceinline__ float real(const void* p, int dtype, int64_t i) {
  if (dtype == BETTY_F32) return ((const float*)p)[i];
  return dtype == BETTY_BF16 ? __bfloat162float(((const __nv_bfloat16*)p)[i]) : __half2float(((const __half*)p)[i]);
}

// ------------------------------------------------------------------ a teacher's entries
// A warp per row: the softmax of the row's logits over T, and its entries in ascending order of (id, place), by a bitonic sort of
// 32-bit keys (22 bits of id, 10 of place) in registers: place 32 r + lane in register r.  An entry without an id of the
// vocabulary or with a logit of -inf is none: what else its logit is is not looked at.  The maximum is taken away before T divides:
// finite logits stay finite, or end as shares of zero, however large they are and however small T.  The same id twice stays two
// entries; their shares add up where they are used.  (Sorted by a block in shared memory: 32 us for 8192 rows of 128.)
struct EntryArgs {
  int64_t rows, vocab;
  const void* ids; int64_t ldi; int id64;
  const void* logits; int64_t ldt; int dtype;
  int top; float c2;                           // log2(e) / T
  int2* out; int64_t out_row, out_place;       // from a row's entries to the next one's, from an entry to the next
  uint8_t* some;
};
static constexpr uint32_t NO_KEY = 0xFFFFFFFFu;
template <int R>
__global__ void __launch_bounds__(256) k_entries(const EntryArgs a) {
  __shared__ float shares[8][32 * R];
  pdl_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t row = (int64_t)blockIdx.x * 8 + warp;
  if (row >= a.rows) return;
  uint32_t key[R];
  float t[R], m = -INFINITY, s = 0.f;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int j = r * 32 + lane;
    key[r] = NO_KEY;
    t[r] = -INFINITY;
    if (j < a.top) {
      const int64_t id = whole(a.ids, a.id64, row * a.ldi + j);
      const float x = real(a.logits, a.dtype, row * a.ldt + j);
      if (id >= 0 && id < a.vocab && x != -INFINITY) {
        key[r] = (uint32_t)id << 10 | (uint32_t)j;
        t[r] = x;
      }
    }
    m = fmaxf(m, t[r]);
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    t[r] = exp2f((t[r] - base) * a.c2);
    s += t[r];
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  const float inv = 1.f / s;
#pragma unroll
  for (int r = 0; r < R; ++r) shares[warp][r * 32 + lane] = t[r] * inv;
#pragma unroll
  for (int size = 2; size <= 32 * R; size <<= 1) {
#pragma unroll
    for (int stride = size >> 1; stride; stride >>= 1) {
      if (stride >= 32) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const int other = r ^ (stride >> 5);
          if (other > r) {
            const bool up = ((r * 32) & size) == 0;
            const uint32_t lo = min(key[r], key[other]), hi = max(key[r], key[other]);
            key[r] = up ? lo : hi;
            key[other] = up ? hi : lo;
          }
        }
      } else {
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const uint32_t other = __shfl_xor_sync(0xffffffffu, key[r], stride);
          const bool up = ((r * 32 + lane) & size) == 0, lower = (lane & stride) == 0;
          key[r] = up == lower ? min(key[r], other) : max(key[r], other);
        }
      }
    }
  }
  __syncwarp();
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int j = r * 32 + lane;
    if (j < a.top) a.out[row * a.out_row + j * a.out_place] = key[r] != NO_KEY ? make_int2((int32_t)(key[r] >> 10), __float_as_int(shares[warp][key[r] & 1023u])) : make_int2(NO_ID, 0);
  }
  if (lane == 0) a.some[row] = key[0] != NO_KEY;
}
template <int R>
static betty_status sort_entries(cudaStream_t stream, const EntryArgs& a) {
  if constexpr (R < 32)
    if (a.top > 32 * R) return sort_entries<2 * R>(stream, a);
  launch_pdl(k_entries<R>, dim3((unsigned)((a.rows + 7) / 8)), dim3(256), 0, stream, a);
  BETTY_LAUNCH_CHECK();
  return BETTY_OK;
}

// ------------------------------------------------------------------ the rows that count
struct RowArgs {
  int64_t rows, vocab;
  int d;
  int64_t dp, ldx;
  const uint16_t* x_in;
  const void* target; int id64; float share;   // cross entropy: an entry (target, share) per row
  const uint8_t* some;                         // distillation: whether a row has an entry
  int2* entry; const int2* entry_in; int top;  // entries in the order of the copies (of entry_in's: distillation)
  int64_t rpad;
  Meta* meta; int32_t* src; int32_t* pos; uint16_t* x; uint16_t* x_dw;
  float* loss; float* lse_out;                 // forward: zeros for rows left out
  const float* lse; const float* dloss;        // backward
  RowCoef* coef; float* row_scale;
  float inv_t, z_loss, smoothing;
  int fp16;
  int lanes, workers, cols, want_dx, want_dw, twice;   // the gradients' products
  int64_t sum_rows;
  AlignRows align; int row_blocks;             // the blocks behind row_blocks copy W to 16-byte boundaries, where that is needed
};

// What says whether a row counts: its target, or whether it has an entry, and its weight
struct Mark { int64_t t; float g; };
__device__ __forceinline__ Mark mark(const RowArgs& a, int64_t i) {
  return {a.some ? (a.some[i] ? 0 : -1) : whole(a.target, a.id64, i), a.dloss ? a.dloss[i] : 1.f};
}
__device__ __forceinline__ bool counts(const RowArgs& a, const Mark& m) { return m.t >= 0 && m.t < a.vocab && !(m.g == 0.f); }
// bound of a row's |dz|
__device__ __forceinline__ float bound_of(const RowArgs& a, int64_t i, float g) {
  return fabsf(g * a.inv_t) * (a.z_loss != 0.f ? 1.f + 2.f * a.z_loss * fabsf(a.lse[i]) : 1.f);
}
// exponent that brings a bound to [2^13, 2^14); of bounds below 2^-113 only to 2^126 times themselves, 1 or more: 2^-126 is the smallest power
// that the way back can multiply by.  Of a bound that is zero or not finite: none
__device__ __forceinline__ int lift(float bound) { return bound > 0.f && bound < INFINITY ? min(13 - ilogbf(bound), 126) : 0; }
static constexpr int NO_LIFT = 1 << 20;
// Half precision: a row's coefficients are stored as dz 2^h, with h from the row's own bound, so that none of a row with a small
// weight is lost; the sums dX take 2^-h back.  dW sums over rows of different h: with H the smallest, x is scaled by
// 2^(H - h) for it.  Rows within 2^6 of the largest bound share H, so that their x is not scaled at all: 2^13 / 2^6 / 128 Ki
// is still a normal number of the type.
__device__ __forceinline__ int row_lift(float bound, int least) {
  const int h = lift(bound);
  return h <= least + 6 ? least : h - 6;
}

// Copies a segment of a row to a 16-byte boundary, zeros behind the row's end; a warp.  scale: 1, or a power of two for the second copy
static constexpr int SEGMENT = 1024;
__device__ __forceinline__ void copy_segment(const RowArgs& a, int64_t from, int64_t to, int segment, float scale) {
  const int lane = threadIdx.x & 31;
  const uint16_t* in = a.x_in + from * a.ldx;
  uint16_t* out = a.x + to * a.dp;
  uint16_t* out2 = a.x_dw != a.x ? a.x_dw + to * a.dp : nullptr;
  uint16_t* again = a.twice ? a.x_dw + (to + TWICE_ROWS) * a.dp : nullptr;
  constexpr int U = SEGMENT / 256;     // accesses in flight
  const int c0 = segment * SEGMENT + lane * 8;
  {
    Words raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = fetch8(in, c0 + 256 * u, a.d);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + 256 * u;
      if (c >= a.dp) break;
      uint4 v = shift8(raw[u], in, c, a.d);
      *(uint4*)(out + c) = v;
      if (out2) {
        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 f = __half22float2(*(__half2*)&w[k]);
          const __half2 h = __floats2half2_rn(f.x * scale, f.y * scale);
          w[k] = *(const uint32_t*)&h;
        }
        v = make_uint4(w[0], w[1], w[2], w[3]);
        *(uint4*)(out2 + c) = v;
      }
      if (again) *(uint4*)(again + c) = v;
    }
  }
}

// Parts of dX's contraction, for which there is room: the number with which the workers finish soonest, where dX's tiles come
// first and dW's fill up.  Times in chunks of a contraction; a part's sums are written and read again.
__device__ int choose_split(const RowArgs& a, int n) {           // a warp
  const Products p = products_of(n, a.d, a.cols, a.lanes);
  const int most = min((int)(a.sum_rows / max(1, p.row_tiles * a.lanes)), max(1, p.dx_chunks / 8));
  const int tiles = p.row_tiles * p.d_tiles;
  // one tile of rows: W streams past it once, and that is the time; all workers take part in it, in one round (24 rows, 32000 x 2048
  // in 3 / 6 / 9 / 12 parts: 98.5 / 92.9 / 91.9 / 95.7 us; 8 rows, 128000 x 4096 in 3 / 4 / 6: 579 / 558 / 619)
  if (p.row_tiles <= 1) return min(most, max(1, a.workers / max(1, tiles)));
  const float second = a.want_dw ? (float)p.col_tiles * p.d_tiles * dw_cost(p) : 0.f;
  const float part = (float)n * a.dp * (a.lanes == 256 ? 3.6e-6f : 7e-6f);      // 8 bytes a value at 6 TB/s, chunks of 0.37 (0.19) us
  int best = 1;
  float least = INFINITY;
  for (int s = 1 + (threadIdx.x & 31); s <= most; s += 32) {
    const float first = (float)((tiles * s + a.workers - 1) / a.workers) * dx_cost(p, s);
    const float time = fmaxf(first, ((float)tiles * s * dx_cost(p, s) + second) / a.workers) + s * part;
    if (time < least) { least = time; best = s; }
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const float t = __shfl_xor_sync(0xffffffffu, least, o);
    const int s = __shfl_xor_sync(0xffffffffu, best, o);
    if (t < least || (t == least && s < best)) { least = t; best = s; }
  }
  return best;
}

// Each block takes a range of rows and counts those before it itself: one launch, and the order is kept.
__global__ void __launch_bounds__(ROW_THREADS) k_rows(const RowArgs a) {
  __shared__ int counted[8], least_of[8];
  __shared__ int list[ROW_THREADS];
  __shared__ float scales[ROW_THREADS];
  pdl_enter();
  if ((int)blockIdx.x >= a.row_blocks) {
    // narrow rows: fewer accesses (as in align.cu, with this kernel's registers): 60000 x 500 and a pass over it 41.5 instead of 45 us
    if (a.align.ld <= 1280) align_rows<3>(a.align, blockIdx.x - a.row_blocks, gridDim.x - a.row_blocks);
    else align_rows<4>(a.align, blockIdx.x - a.row_blocks, gridDim.x - a.row_blocks);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t r0 = a.rows * blockIdx.x / a.row_blocks, r1 = a.rows * (blockIdx.x + 1) / a.row_blocks;
  int before = 0, least = NO_LIFT;
  const bool lifted = a.fp16 && a.dloss;
  const int64_t seen = lifted ? a.rows : r0;
  constexpr int U = 8;                 // rows in flight
  for (int64_t i0 = tid; i0 < seen; i0 += ROW_THREADS * U) {
    Mark m[U];
#pragma unroll
    for (int u = 0; u < U; ++u) m[u] = i0 + u * ROW_THREADS < seen ? mark(a, i0 + u * ROW_THREADS) : Mark{-1, 0.f};
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (counts(a, m[u])) {
        const int64_t i = i0 + u * ROW_THREADS;
        before += i < r0;
        if (lifted) {
          const float b = bound_of(a, i, m[u].g);
          if (b > 0.f && b < INFINITY) least = min(least, lift(b));
        }
      }
  }
  before = __reduce_add_sync(0xffffffffu, before);
  least = __reduce_min_sync(0xffffffffu, least);
  if (lane == 0) { counted[warp] = before; least_of[warp] = least; }
  __syncthreads();
  before = 0;
  for (int i = 0; i < 8; ++i) { before += counted[i]; least = min(least, least_of[i]); }
  if (least == NO_LIFT) least = 0;
  for (int64_t base = r0; base < r1; base += ROW_THREADS) {
    __syncthreads();                   // counted and list are free again
    const int64_t i = base + tid;
    const Mark m = i < r1 ? mark(a, i) : Mark{-1, 0.f};
    const float lse = a.dloss && i < r1 ? a.lse[i] : 0.f;
    const bool live = counts(a, m);
    const uint32_t votes = __ballot_sync(0xffffffffu, live);
    if (lane == 0) counted[warp] = __popc(votes);
    __syncthreads();
    int at = 0, all = 0;
    for (int k = 0; k < 8; ++k) { if (k < warp) at += counted[k]; all += counted[k]; }
    at += __popc(votes & ((1u << lane) - 1u));
    if (i < r1) {
      a.pos[i] = live ? before + at : -1;
      if (live) {
        const int64_t to = before + at;
        list[at] = (int)(i - base);
        a.src[to] = (int32_t)i;
        if (!a.some) a.entry[to] = make_int2((int32_t)m.t, __float_as_int(a.share));
        if (a.dloss) {
          const int h = a.fp16 ? row_lift(bound_of(a, i, m.g), least) : 0;
          const float g = ldexpf(m.g * a.inv_t, h);
          scales[at] = ldexpf(1.f, least - h);
          a.coef[to] = {lse * LOG2E, g * (1.f + 2.f * a.z_loss * lse), -g * a.smoothing / (float)a.vocab, g};
          a.row_scale[to] = ldexpf(1.f, -h);
        }
      } else if (a.loss) {
        a.loss[i] = 0.f;
        a.lse_out[i] = 0.f;
      }
    }
    __syncthreads();
    if (a.some)
      for (int k = tid; k < all * a.top; k += ROW_THREADS) {
        const int j = k / all, r = k - j * all;
        a.entry[j * a.rpad + before + r] = a.entry_in[(base + list[r]) * a.top + j];
      }
    const int segments = (int)((a.dp + SEGMENT - 1) / SEGMENT);
    for (int k = warp; k < all * segments; k += 8) {
      const int r = k / segments;
      copy_segment(a, base + list[r], before + r, k - r * segments, lifted ? scales[r] : 1.f);
    }
    before += all;
  }
  if ((int)blockIdx.x == a.row_blocks - 1) {
    if (warp == 0) {
      const int split = a.dloss && a.want_dx ? choose_split(a, before) : 1;
      if (lane == 0) { a.meta->n = before; a.meta->split = split; a.meta->dw_scale = lifted ? ldexpf(1.f, -least) : 1.f; }
    }
    if (a.dloss) {                     // a contraction over the rows takes them 16 at a time, or all that there is room for, twice
      const int end = a.twice ? TWICE_ROWS : (before + 15) / 16 * 16, copies = a.twice ? 2 : 1;
      for (int r = before + warp; r < end; r += 8)
        for (int c = lane * 8; c < a.dp; c += 256)
          for (int k = 0; k < copies; ++k) *(uint4*)(a.x_dw + (int64_t)(r + k * TWICE_ROWS) * a.dp + c) = make_uint4(0u, 0u, 0u, 0u);
    }
  }
}

// ------------------------------------------------------------------ losses
struct LossArgs {
  const Meta* meta; const int32_t* src;
  const float2* part; const float* part_y; int parts; int64_t rpad;
  const int2* entry; const float* y_entry; int top;
  int distill;
  float smoothing, z_loss; int64_t vocab;
  float* loss; float* lse;
  // x in place: so many rows, each in its own place; which of them count
  int rows; const void* target; int id64; const uint8_t* some; float share;
};
// A sum that takes along what its additions round away: a thread adds up to 2048 parts (2^22 columns in half tiles of 128, 16 threads a
// row), and parts that all round the same way would end 2^-15 off.  With it no sum of powers is a chain of more than 64 additions.  It is
// taken once for the parts in flight, 16 of them in the 32-row form: part by part, eight in flight, 600 rows of 1000 parts took 6 us more.
struct LongSum {
  float s, lost;
  __device__ __forceinline__ void scale(float f) { s *= f; lost *= f; }
  __device__ __forceinline__ void add(float v) {
    const float w = __fsub_rn(v, lost), t = __fadd_rn(s, w);
    lost = __fsub_rn(__fsub_rn(t, s), w);
    s = t;
  }
};
// ROWS rows a block of 512 threads, which share a row's parts and entries: 32 rows for whole cache lines, 8 where there are few.
// Measured, with fewer parts in flight than now: 8192 rows of 512 parts: 14.5 us with 32 (now 10.4), 29 with 8; 8 rows of 572: 14 with 32.
static constexpr int LOSS_THREADS = 512;
template <int ROWS>
__global__ void __launch_bounds__(LOSS_THREADS) k_losses(const LossArgs a) {
  constexpr int SLICES = LOSS_THREADS / ROWS, WARPS = LOSS_THREADS / 32;
  __shared__ float sm[WARPS][ROWS], ss[WARPS][ROWS], sy[WARPS][ROWS], se[WARPS][ROWS];
  pdl_enter();
  const int col = threadIdx.x % ROWS, slice = threadIdx.x / ROWS, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row = blockIdx.x * ROWS + col, n = a.rows ? a.rows : a.meta->n;
  // few rows: what may be needed is asked for before it is known which rows count (the arrays have room for all)
  constexpr bool EARLY = ROWS == 8;
  if (!EARLY && blockIdx.x * ROWS >= n) return;
  bool live = row < n;
  const bool ask = EARLY || live;
  float m = -INFINITY, s = 0.f, y = 0.f;
  LongSum sum = {0.f, 0.f}, sum_y = {0.f, 0.f};
  // the first of a thread's entries is asked for before the parts
  const int64_t src = a.rows ? row : (ask ? a.src[row] : 0);
  float p0 = 0.f, y0 = 0.f;
  if (ask && slice < a.top) {
    p0 = a.rows && !a.distill ? a.share : __int_as_float(a.entry[slice * a.rpad + row].y);
    y0 = a.y_entry[slice * a.rpad + row];
  }
  bool left_out = false;
  if (a.rows && live) {
    const int64_t t = a.distill ? (int64_t)a.some[row] - 1 : whole(a.target, a.id64, row);
    left_out = t < 0 || t >= a.vocab;
    live = !left_out;
  }
  if (ask) {
    constexpr int U = EARLY ? 12 : 16; // parts in flight
    for (int i0 = slice; i0 < a.parts; i0 += SLICES * U) {
      float2 q[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * SLICES;
        q[u] = i < a.parts ? a.part[(int64_t)i * a.rpad + row] : make_float2(-INFINITY, 0.f);
      }
      float most = m;
#pragma unroll
      for (int u = 0; u < U; ++u) most = fmaxf(most, q[u].x);
      const float base = most == -INFINITY ? 0.f : most;
      float e = 0.f;                   // of the parts in flight: plain additions, U at most one after the other
#pragma unroll
      for (int u = 0; u < U; ++u) e += q[u].y * exp2f(q[u].x - base);
      sum.scale(exp2f(m - base));
      sum.add(e);
      m = most;
    }
    if (a.part_y)
      for (int i0 = slice; i0 < a.parts; i0 += SLICES * 8) {
        float e = 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int i = i0 + u * SLICES;
          e += i < a.parts ? a.part_y[(int64_t)i * a.rpad + row] : 0.f;
        }
        sum_y.add(e);
      }
    s = sum.s;
    y = sum_y.s;
  }
#pragma unroll
  for (int o = ROWS; o < 32; o <<= 1) {
    const float m2 = __shfl_xor_sync(0xffffffffu, m, o), s2 = __shfl_xor_sync(0xffffffffu, s, o), most = fmaxf(m, m2);
    const float base = most == -INFINITY ? 0.f : most, mine = s * exp2f(m - base), other = s2 * exp2f(m2 - base);
    s = mine + other;
    m = most;
    y += __shfl_xor_sync(0xffffffffu, y, o);
  }
  if (lane < ROWS) { sm[warp][col] = m; ss[warp][col] = s; sy[warp][col] = y; }
  __syncthreads();
  float most = -INFINITY;
#pragma unroll
  for (int i = 0; i < WARPS; ++i) most = fmaxf(most, sm[i][col]);
  const float base = most == -INFINITY ? 0.f : most;
  s = y = 0.f;
#pragma unroll
  for (int i = 0; i < WARPS; ++i) { s += ss[i][col] * exp2f(sm[i][col] - base); y += sy[i][col]; }
  const float lse2 = base + log2f(s);
  float e = 0.f;
  if (live)
    for (int i = slice; i < a.top; i += SLICES) {
      const float p = i == slice ? p0 : __int_as_float(a.entry[i * a.rpad + row].y), at = i == slice ? y0 : a.y_entry[i * a.rpad + row];
      // log p - (y - lse2): close to each other where the student has learnt its teacher
      if (p > 0.f) e += p * ((a.distill ? log2f(p) : 0.f) - (at - lse2));
      else if (!(p == 0.f)) e = p;
    }
#pragma unroll
  for (int o = ROWS; o < 32; o <<= 1) e += __shfl_xor_sync(0xffffffffu, e, o);
  if (lane < ROWS) se[warp][col] = e;
  __syncthreads();
  if (slice == 0 && live) {
    e = 0.f;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) e += se[i][col];
    const float lse = lse2 * LN2;
    if (a.smoothing != 0.f) e += a.smoothing * (lse2 - y / (float)a.vocab);
    a.loss[src] = e * LN2 + a.z_loss * lse * lse;
    a.lse[src] = lse;
  } else if (slice == 0 && left_out) {
    a.loss[src] = 0.f;
    a.lse[src] = 0.f;
  }
}

// ------------------------------------------------------------------ dX
// Row i of dX from the parts' sums of its copy, or zeros: blockDim.x threads take `width` columns of a row, four at a time each,
// blockDim.y of them in a block of 256.
template <typename T>
__global__ void __launch_bounds__(256) k_dx(int64_t rows, int d, int64_t dp, int lanes, int width, int twice, const Meta* meta, const int32_t* pos, const float* row_scale,
                                            const float* sums, T* dx, int64_t ld) {
  pdl_enter();
  const bool wide = ((uintptr_t)dx % (4 * sizeof(T))) == 0 && ld % 4 == 0;
  const int strips = (d + width - 1) / width, split = meta->split, step = (int)blockDim.x * 4;
  const int64_t stride = (int64_t)((meta->n + lanes - 1) / lanes * lanes) * dp;
  for (int64_t b = (int64_t)blockIdx.x * blockDim.y + threadIdx.y; b < rows * strips; b += (int64_t)gridDim.x * blockDim.y) {
    const int64_t row = b / strips;
    const int c0 = (int)(b - row * strips) * width, end = min(d, c0 + width);
    const int at = pos[row];
    const float f = at >= 0 ? row_scale[at] : 0.f;
    const float* in = sums + (int64_t)max(at, 0) * dp;
    T* out = dx + row * ld;
#pragma unroll 4
    for (int c = c0 + (int)threadIdx.x * 4; c < end; c += step) {
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (at >= 0) {
        v = *(const float4*)(in + c);
        if (twice) {                   // the remainders' sums first: they are small
          v = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int s = 0; s < split; ++s) {
            const float4 w = *(const float4*)(in + TWICE_ROWS * dp + s * stride + c);
            v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
          }
          const float4 w = *(const float4*)(in + c);
          v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
        }
#pragma unroll 8
        for (int s = 1; s < split; ++s) {
          const float4 w = *(const float4*)(in + s * stride + c);
          v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
        }
        v.x *= f; v.y *= f; v.z *= f; v.w *= f;
      }
      if (wide && c + 4 <= d) {
        alignas(16) T o[4] = {from_f<T>(v.x), from_f<T>(v.y), from_f<T>(v.z), from_f<T>(v.w)};
        if constexpr (sizeof(T) == 4) *(float4*)(out + c) = *(const float4*)o;
        else *(uint2*)(out + c) = *(const uint2*)o;
      } else {
        const float o[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (c + k < d) out[c + k] = from_f<T>(o[k]);
      }
    }
  }
}

__global__ void __launch_bounds__(256) k_zero_rows(int64_t rows, int d, unsigned char* p, int64_t ld, int bytes) {
  pdl_enter();
  for (int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); row < rows; row += (int64_t)gridDim.x * 8)
    for (int64_t c = threadIdx.x & 31; c < d; c += 32) {
      if (bytes == 4) ((float*)p)[row * ld + c] = 0.f;
      else ((uint16_t*)p)[row * ld + c] = 0;
    }
}

// ------------------------------------------------------------------ host side
static int64_t round_up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

struct Call {
  const betty_vocab_cfg* cfg;
  int64_t rows;
  const void* X; int64_t ldx;
  const void* W; int64_t ldw;
  const void* target; int32_t id_dtype;
  int top; int64_t ldi;                        // distillation: top >= 1, else 0
  const void* teacher; int64_t ldt; int32_t teacher_dtype;
  float* loss; float* lse_out;                 // forward
  const float* lse; const float* dloss;        // backward
  void* dX; int64_t lddx; int32_t dx_dtype;
  void* dW; int64_t lddw; int32_t dw_dtype;
  bool backward;
};

static betty_status check_cfg(const betty_vocab_cfg* c, int64_t rows, int64_t top) {
  if (!c || rows < 0) return BETTY_ERR_INVALID_ARG;
  if (c->dtype != BETTY_BF16 && c->dtype != BETTY_F16) return BETTY_ERR_DTYPE;
  if (c->vocab < 1 || c->d < 1 || top < 0) return BETTY_ERR_SHAPE;
  // 32-bit tile counts and coordinates; 32-bit keys of (id, place)
  if (c->vocab >= (1 << 22) || c->d > (1 << 16) || rows > (1 << 22) || top > MAX_TOP) return BETTY_ERR_UNSUPPORTED;
  if (!(c->temperature > 0.f) || !(c->temperature <= 1e30f) || !(c->temperature >= 1e-30f)) return BETTY_ERR_INVALID_ARG;
  if (!(c->smoothing >= 0.f) || !(c->smoothing <= 1.f) || !(c->z_loss >= 0.f) || !(c->z_loss <= 1e30f)) return BETTY_ERR_INVALID_ARG;
  return BETTY_OK;
}
static betty_status check_matrix(const void* p, int64_t ld, int64_t rows, int64_t cols, int64_t bytes) {
  if (!p) return BETTY_ERR_INVALID_ARG;
  if (rows > 1 && ld < cols) return BETTY_ERR_SHAPE;
  if (ld > ((int64_t)1 << 32)) return BETTY_ERR_UNSUPPORTED;      // 40-bit strides of tensor maps
  return (uintptr_t)p % bytes ? BETTY_ERR_ALIGNMENT : BETTY_OK;
}
static int64_t float_bytes(int dtype) { return dtype == BETTY_F32 ? 4 : (dtype == BETTY_BF16 || dtype == BETTY_F16 ? 2 : 0); }

static betty_status check(const Call& c, void* ws, size_t ws_bytes) {
  BETTY_TRY(check_cfg(c.cfg, c.rows, c.top));
  const bool distill = c.teacher_dtype >= 0;
  if (distill && c.top < 1) return BETTY_ERR_SHAPE;
  if (distill && (c.cfg->smoothing != 0.f || c.cfg->z_loss != 0.f)) return BETTY_ERR_UNSUPPORTED;
  if (c.id_dtype != BETTY_I32 && c.id_dtype != BETTY_I64) return BETTY_ERR_DTYPE;
  if (distill && !float_bytes(c.teacher_dtype)) return BETTY_ERR_DTYPE;
  if (c.backward) {
    if (c.rows && !c.dX && !c.dW) return BETTY_ERR_INVALID_ARG;   // of no rows dX has no values and may have no address
    if (c.dX && c.dx_dtype != BETTY_F32 && c.dx_dtype != c.cfg->dtype) return BETTY_ERR_DTYPE;
    if (c.dW && c.dw_dtype != BETTY_F32 && c.dw_dtype != c.cfg->dtype) return BETTY_ERR_DTYPE;
  }
  if (!ws || ws_bytes < sizeof(StatusBlock) || (((uintptr_t)ws) & 255u)) return BETTY_ERR_WORKSPACE;
  if (c.dW) BETTY_TRY(check_matrix(c.dW, c.lddw, c.cfg->vocab, c.cfg->d, float_bytes(c.dw_dtype)));
  if (c.rows == 0) return BETTY_OK;
  BETTY_TRY(check_matrix(c.X, c.ldx, c.rows, c.cfg->d, 2));
  BETTY_TRY(check_matrix(c.W, c.ldw, c.cfg->vocab, c.cfg->d, 2));
  if (c.dX) BETTY_TRY(check_matrix(c.dX, c.lddx, c.rows, c.cfg->d, float_bytes(c.dx_dtype)));
  const int64_t ib = c.id_dtype == BETTY_I64 ? 8 : 4;
  if (distill) {
    BETTY_TRY(check_matrix(c.target, c.ldi, c.rows, c.top, ib));
    BETTY_TRY(check_matrix(c.teacher, c.ldt, c.rows, c.top, float_bytes(c.teacher_dtype)));
  } else {
    BETTY_TRY(check_matrix(c.target, 1, 1, 1, ib));
  }
  const float* vectors[4] = {c.backward ? c.lse : c.loss, c.backward ? c.dloss : c.lse_out, nullptr, nullptr};
  for (int i = 0; i < 2; ++i) BETTY_TRY(check_matrix(vectors[i], 1, 1, 1, 4));
  return BETTY_OK;
}

static Shape shape_of(const betty_vocab_cfg* c, int64_t rows, int top, bool backward, bool dx, bool dw) {
  Shape s = {};
  s.dtype = c->dtype; s.rows = (int)rows; s.rpad = round_up(rows < 1 ? 1 : rows, 256);
  s.vocab = (int)c->vocab; s.d = (int)c->d; s.dp = round_up(c->d, 64);
  s.c2 = LOG2E / c->temperature;
  s.top = top < 1 ? 1 : top;
  s.want_dx = dx; s.want_dw = dw;
  choose_shape(s, backward);
  return s;
}

// The call's arrays; with an empty arena: only their size.
static betty_status lay_out(Arena& arena, const Shape& s, const Call& c, Buffers& b, uint8_t*& some) {
  const bool distill = c.teacher_dtype >= 0;
  b.sb = arena.status();
  b.meta = arena.alloc<Meta>(1);
  b.src = arena.alloc<int32_t>((size_t)s.rpad);
  b.pos = arena.alloc<int32_t>((size_t)c.rows);
  b.entry = arena.alloc<int2>((size_t)(s.rpad * s.top));
  b.entry_in = distill ? arena.alloc<int2>((size_t)(c.rows * s.top)) : nullptr;
  some = distill ? arena.alloc<uint8_t>((size_t)c.rows) : nullptr;
  b.x = b.x_dw = arena.alloc<uint16_t>((size_t)(s.rpad * s.dp));
  b.part = nullptr; b.part_y = b.y_entry = nullptr; b.coef = nullptr; b.row_scale = nullptr; b.dz = nullptr; b.dx = nullptr;
  if (!c.backward) {
    const int64_t parts = logits_parts(s);
    b.part = arena.alloc<float2>((size_t)(parts * s.rpad));
    if (c.cfg->smoothing != 0.f) b.part_y = arena.alloc<float>((size_t)(parts * s.rpad));
    b.y_entry = arena.alloc<float>((size_t)(s.rpad * s.top));
  } else {
    b.coef = arena.alloc<RowCoef>((size_t)s.rpad);
    b.row_scale = arena.alloc<float>((size_t)s.rpad);
    b.dz = arena.alloc<uint16_t>((size_t)(s.rpad * s.piece));
    if (c.dX) b.dx = arena.alloc<float>((size_t)(s.sum_rows * s.dp));
    if (c.dW && s.dtype == BETTY_F16) b.x_dw = arena.alloc<uint16_t>((size_t)(s.rpad * s.dp));
  }
  return arena.overflow ? BETTY_ERR_WORKSPACE : BETTY_OK;
}

static betty_status evaluate(const Call& c, void* ws, size_t ws_bytes, void* stream_) {
  BETTY_TRY(check(c, ws, ws_bytes));
  const cudaStream_t stream = (cudaStream_t)stream_;
  const betty_vocab_cfg* cfg = c.cfg;
  const int64_t most = (int64_t)current_sm_count() * 4;
  if (c.rows == 0) {
    if (!c.dW) return BETTY_OK;
    launch_pdl(k_zero_rows, dim3((unsigned)most), dim3(256), 0, stream, cfg->vocab, (int)cfg->d, (unsigned char*)c.dW, c.lddw, c.dw_dtype == BETTY_F32 ? 4 : 2);
    BETTY_LAUNCH_CHECK();
    return BETTY_OK;
  }
  const bool distill = c.teacher_dtype >= 0;
  const Shape s = shape_of(cfg, c.rows, c.top, c.backward, c.dX != nullptr, c.dW != nullptr);
  Arena arena(ws, ws_bytes);
  Buffers b = {};
  uint8_t* some;
  BETTY_TRY(lay_out(arena, s, c, b, some));
  Operand w = {c.W, cfg->d, cfg->vocab, 1, c.ldw, 0};
  RowArgs r = {};
  BETTY_TRY(plan_alignment(arena, w, r.align));
  const int64_t ldx = c.rows == 1 ? pad8(cfg->d) : c.ldx;
  const bool in_place = !c.backward && c.rows <= IN_PLACE_ROWS && aligned16(c.X) && ldx % 8 == 0 && !r.align.rows;
  if (distill) {
    const EntryArgs e = {c.rows, cfg->vocab, c.target, c.ldi, c.id_dtype == BETTY_I64, c.teacher, c.ldt, c.teacher_dtype, c.top, s.c2, in_place ? b.entry : b.entry_in,
                         in_place ? 1 : c.top, in_place ? s.rpad : 1, some};
    BETTY_TRY(sort_entries<1>(stream, e));
  }
  LossArgs l = {};
  if (!c.backward) {
    l.meta = b.meta; l.src = b.src; l.part = b.part; l.part_y = b.part_y; l.parts = logits_parts(s); l.rpad = s.rpad;
    l.entry = b.entry; l.y_entry = b.y_entry; l.top = s.top; l.distill = distill;
    l.smoothing = cfg->smoothing; l.z_loss = cfg->z_loss; l.vocab = cfg->vocab; l.loss = c.loss; l.lse = c.lse_out;
  }
  const int id64 = c.id_dtype == BETTY_I64;
  const float share = 1.f - cfg->smoothing;
  if (in_place) {
    const InPlace p = {c.X, ldx, distill ? nullptr : c.target, id64, share};
    BETTY_TRY(logits_statistics(stream, s, b, w, true, &p));
    l.rows = (int)c.rows; l.target = c.target; l.id64 = id64; l.some = some; l.share = share;
    launch_pdl(k_losses<8>, dim3((unsigned)((c.rows + 7) / 8)), dim3(LOSS_THREADS), 0, stream, l);
    BETTY_LAUNCH_CHECK();
    return BETTY_OK;
  }
  r.rows = c.rows; r.vocab = cfg->vocab; r.d = (int)cfg->d; r.dp = s.dp; r.ldx = c.ldx; r.x_in = (const uint16_t*)c.X;
  r.target = distill ? nullptr : c.target; r.id64 = id64; r.share = share; r.some = some;
  r.entry = b.entry; r.entry_in = b.entry_in; r.top = s.top; r.rpad = s.rpad;
  r.meta = b.meta; r.src = b.src; r.pos = b.pos; r.x = b.x; r.x_dw = b.x_dw;
  r.loss = c.backward ? nullptr : c.loss; r.lse_out = c.lse_out; r.lse = c.lse; r.dloss = c.backward ? c.dloss : nullptr;
  r.coef = b.coef; r.row_scale = b.row_scale;
  r.inv_t = 1.f / cfg->temperature; r.z_loss = cfg->z_loss; r.smoothing = cfg->smoothing; r.fp16 = cfg->dtype == BETTY_F16;
  r.lanes = s.product_pairs ? 256 : 128; r.workers = current_sm_count() / (s.product_pairs ? 2 : 1);
  r.cols = s.piece < s.vocab ? s.piece : s.vocab; r.want_dx = s.want_dx; r.want_dw = s.want_dw; r.twice = s.twice; r.sum_rows = s.sum_rows;
  // a block a row where there are few (the warps share it), about four rows a block up to four blocks an SM
  const int64_t sms = current_sm_count(), fours = (c.rows + 3) / 4, blocks = fours < sms ? (c.rows < sms ? c.rows : sms) : fours;
  r.row_blocks = (int)(blocks < most ? blocks : most);
  launch_pdl(k_rows, dim3((unsigned)(r.row_blocks + (r.align.rows ? align_blocks(r.align) : 0))), dim3(ROW_THREADS), 0, stream, r);
  BETTY_LAUNCH_CHECK();
  const bool copied = r.align.rows != 0;

  if (!c.backward) {
    BETTY_TRY(logits_statistics(stream, s, b, w, !copied, nullptr));
    if (c.rows <= 512) launch_pdl(k_losses<8>, dim3((unsigned)((c.rows + 7) / 8)), dim3(LOSS_THREADS), 0, stream, l);
    else launch_pdl(k_losses<32>, dim3((unsigned)((c.rows + 31) / 32)), dim3(LOSS_THREADS), 0, stream, l);
    BETTY_LAUNCH_CHECK();
    return BETTY_OK;
  }
  BETTY_TRY(logits_gradients(stream, s, b, w, !copied, c.dW, c.lddw, c.dw_dtype));
  if (c.dX) {
    // a row's threads: four accesses of four columns each; few rows: one access, and more blocks than rows
    const int accesses = c.rows < most ? 1 : 4;
    int across = 32;
    while (across < 256 && across * 4 * accesses < cfg->d) across *= 2;
    const int width = c.rows < most ? across * 4 : (int)s.dp;
    const int64_t strips = (c.rows * ((cfg->d + width - 1) / width) + 256 / across - 1) / (256 / across);
    const dim3 grid((unsigned)(strips < most * 2 ? strips : most * 2)), block((unsigned)across, (unsigned)(256 / across));
    if (c.dx_dtype == BETTY_F32)
      launch_pdl(k_dx<float>, grid, block, 0, stream, c.rows, (int)cfg->d, s.dp, r.lanes, width, s.twice, b.meta, b.pos, b.row_scale, b.dx, (float*)c.dX, c.lddx);
    else if (c.dx_dtype == BETTY_BF16)
      launch_pdl(k_dx<__nv_bfloat16>, grid, block, 0, stream, c.rows, (int)cfg->d, s.dp, r.lanes, width, s.twice, b.meta, b.pos, b.row_scale, b.dx, (__nv_bfloat16*)c.dX, c.lddx);
    else
      launch_pdl(k_dx<__half>, grid, block, 0, stream, c.rows, (int)cfg->d, s.dp, r.lanes, width, s.twice, b.meta, b.pos, b.row_scale, b.dx, (__half*)c.dX, c.lddx);
    BETTY_LAUNCH_CHECK();
  }
  return BETTY_OK;
}

// What any call on up to `rows` rows needs.  The tiles go by the number of 128-row tiles: a call on fewer rows can need more than one
// on all of them.
static size_t workspace_bytes(const betty_vocab_cfg* cfg, int64_t rows, int top, bool any_layout) {
  size_t most = 0;
  for (int64_t tiles = 1; tiles <= (rows < 1 ? 1 : (rows + 127) / 128); ++tiles)
    for (int form = 0; form < 4; ++form) {       // forward; gradients of x and W, of x, of W
      Call c = {};
      c.cfg = cfg; c.rows = rows < tiles * 128 ? rows : tiles * 128; c.top = top; c.teacher_dtype = top > 0 ? BETTY_F32 : -1;
      c.backward = form > 0;
      c.dX = form == 1 || form == 2 ? &c : nullptr;
      c.dW = form == 1 || form == 3 ? &c : nullptr;
      Arena arena((void*)256, SIZE_MAX / 2);
      Buffers b = {};
      uint8_t* some;
      (void)lay_out(arena, shape_of(cfg, c.rows, top, c.backward, c.dX != nullptr, c.dW != nullptr), c, b, some);
      if (arena.off > most) most = arena.off;
    }
  return most + (any_layout ? 256 + (size_t)(cfg->vocab * pad8(cfg->d)) * 2 : 0);
}

}  // namespace vocab
}  // namespace betty

using namespace betty;

extern "C" betty_status betty_vocab_workspace_size(const betty_vocab_cfg* cfg, int64_t rows, int32_t top, int32_t any_layout, size_t* bytes) {
  if (!bytes) return BETTY_ERR_INVALID_ARG;
  BETTY_TRY(vocab::check_cfg(cfg, rows, top));
  *bytes = vocab::workspace_bytes(cfg, rows, top, any_layout != 0);
  return BETTY_OK;
}

extern "C" betty_status betty_vocab_ce(const betty_vocab_cfg* cfg, int64_t rows, const void* X, int64_t ldx, const void* W, int64_t ldw, const void* target,
                                       int32_t target_dtype, float* loss, float* lse, void* ws, size_t ws_bytes, void* stream) {
  vocab::Call c = {};
  c.cfg = cfg; c.rows = rows; c.X = X; c.ldx = ldx; c.W = W; c.ldw = ldw; c.target = target; c.id_dtype = target_dtype; c.teacher_dtype = -1;
  c.loss = loss; c.lse_out = lse;
  return vocab::evaluate(c, ws, ws_bytes, stream);
}

extern "C" betty_status betty_vocab_ce_backward(const betty_vocab_cfg* cfg, int64_t rows, const void* X, int64_t ldx, const void* W, int64_t ldw,
                                                const void* target, int32_t target_dtype, const float* lse, const float* dloss, void* dX, int64_t lddx,
                                                int32_t dx_dtype, void* dW, int64_t lddw, int32_t dw_dtype, void* ws, size_t ws_bytes, void* stream) {
  vocab::Call c = {};
  c.cfg = cfg; c.rows = rows; c.X = X; c.ldx = ldx; c.W = W; c.ldw = ldw; c.target = target; c.id_dtype = target_dtype; c.teacher_dtype = -1;
  c.lse = lse; c.dloss = dloss; c.dX = dX; c.lddx = lddx; c.dx_dtype = dx_dtype; c.dW = dW; c.lddw = lddw; c.dw_dtype = dw_dtype; c.backward = true;
  return vocab::evaluate(c, ws, ws_bytes, stream);
}

extern "C" betty_status betty_vocab_distill(const betty_vocab_cfg* cfg, int64_t rows, const void* X, int64_t ldx, const void* W, int64_t ldw, int32_t top,
                                            const void* ids, int64_t ldi, int32_t id_dtype, const void* teacher, int64_t ldt, int32_t teacher_dtype,
                                            float* loss, float* lse, void* ws, size_t ws_bytes, void* stream) {
  vocab::Call c = {};
  if (teacher_dtype < 0) return BETTY_ERR_DTYPE;
  c.cfg = cfg; c.rows = rows; c.X = X; c.ldx = ldx; c.W = W; c.ldw = ldw; c.target = ids; c.id_dtype = id_dtype; c.top = top; c.ldi = ldi;
  c.teacher = teacher; c.ldt = ldt; c.teacher_dtype = teacher_dtype; c.loss = loss; c.lse_out = lse;
  return vocab::evaluate(c, ws, ws_bytes, stream);
}

extern "C" betty_status betty_vocab_distill_backward(const betty_vocab_cfg* cfg, int64_t rows, const void* X, int64_t ldx, const void* W, int64_t ldw,
                                                     int32_t top, const void* ids, int64_t ldi, int32_t id_dtype, const void* teacher, int64_t ldt,
                                                     int32_t teacher_dtype, const float* lse, const float* dloss, void* dX, int64_t lddx, int32_t dx_dtype,
                                                     void* dW, int64_t lddw, int32_t dw_dtype, void* ws, size_t ws_bytes, void* stream) {
  vocab::Call c = {};
  if (teacher_dtype < 0) return BETTY_ERR_DTYPE;
  c.cfg = cfg; c.rows = rows; c.X = X; c.ldx = ldx; c.W = W; c.ldw = ldw; c.target = ids; c.id_dtype = id_dtype; c.top = top; c.ldi = ldi;
  c.teacher = teacher; c.ldt = ldt; c.teacher_dtype = teacher_dtype; c.lse = lse; c.dloss = dloss;
  c.dX = dX; c.lddx = lddx; c.dx_dtype = dx_dtype; c.dW = dW; c.lddw = lddw; c.dw_dtype = dw_dtype; c.backward = true;
  return vocab::evaluate(c, ws, ws_bytes, stream);
}
