// Norms before and after a residual block, fused with its gate and residual scale.
//
//   m = N_post(y)      z = m * w_post (+ b_post)      x' = x + s * a(g) * z      u = N_pre(x') * w_pre (+ b_pre)
//
// N is the identity, the RMS norm  v / sqrt(mean(v^2) + eps)  or the layer norm (the same of v - mean(v)); a is 1, the
// gate itself or its sigmoid.  The shared pieces of the forward and the backward kernel: how a row is laid over
// threads, how rows are fetched ahead, and the sums over a row.
#pragma once
#include "common.cuh"

namespace betty {
namespace blocknorm {

// A row is held by G threads (a power of two, 32 .. MAX_G), CH * 8 values each, in granules of GR consecutive values that
// every stream's layout lets a thread copy by itself: 8 where rows start on 16-byte boundaries, 2 where they start on 4-byte
// boundaries (16-bit values), 1 elsewhere.  Neighbouring threads hold neighbouring granules.
static constexpr int MAX_G = 512;
static constexpr int MAX_CH = 4;
static constexpr int MAX_D = MAX_G * 8 * MAX_CH;
static constexpr int SMALL_THREADS = 256;     // block size when a warp holds a row
static constexpr int MAX_STREAMS = 5;

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f(float v) { return v; }
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f(float v) { return __float2half_rn(v); }

// column of a thread's value k (0 .. 7) of chunk c
template <int GR>
__device__ __forceinline__ int column(int c, int k, int t, int G) {
  return ((c * (8 / GR) + k / GR) * G + t) * GR + k % GR;
}

template <typename T> struct alignas(16) Raw8 { T v[8]; };

// chunk c of a row in global memory; columns beyond d are 0
template <int GR, typename T>
__device__ __forceinline__ void load8(float (&o)[8], const T* row, int c, int t, int G, int d) {
  if (GR == 8) {
    Raw8<T> r;
    const int j = (c * G + t) * 8;
    if (j < d) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) ((uint4*)r.v)[i] = *(const uint4*)((const char*)(row + j) + 16 * i);
    } else {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) ((uint4*)r.v)[i] = make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) o[k] = to_f(r.v[k]);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int j = column<GR>(c, k, t, G);
      o[k] = j < d ? to_f(row[j]) : 0.f;
    }
  }
}
template <int GR, typename T>
__device__ __forceinline__ void store8(T* row, const float (&v)[8], int c, int t, int G, int d) {
  if (GR == 8) {
    const int j = (c * G + t) * 8;
    if (j < d) {
      Raw8<T> r;
#pragma unroll
      for (int k = 0; k < 8; ++k) r.v[k] = from_f<T>(v[k]);
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) *(uint4*)((char*)(row + j) + 16 * i) = ((const uint4*)r.v)[i];
    }
  } else if (GR == 2 && sizeof(T) == 2) {
#pragma unroll
    for (int k = 0; k < 8; k += 2) {             // rows start on 4-byte boundaries and d is even
      const int j = column<GR>(c, k, t, G);
      if (j < d) {
        struct alignas(4) Pair { T a, b; } p = {from_f<T>(v[k]), from_f<T>(v[k + 1])};
        *(uint32_t*)(row + j) = *(const uint32_t*)&p;
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int j = column<GR>(c, k, t, G);
      if (j < d) row[j] = from_f<T>(v[k]);
    }
  }
}
// parameters are fp32 and every block of them starts on a 16-byte boundary only when d is a multiple of 4
template <int GR>
__device__ __forceinline__ void load_param8(float (&v)[8], const float* row, int c, int t, int G, int d) { load8<GR, float>(v, row, c, t, G, d); }

// ---- rows fetched ahead ----
// Each thread copies the granules that it will itself read into its own slots of shared memory with cp.async (16 or 4
// bytes at a time), a few rows before their use: no registers are held by data in flight, and as nobody reads another
// thread's slots, waiting for one's own copies is all the synchronisation there is.
// A slot holds CH * 8 values of every stream, interleaved over the G threads so that a warp's accesses are contiguous.
template <int GR, int CH, typename T>
__device__ __forceinline__ void copy_row(char* slot, const T* row, int t, int G, int d) {
  constexpr int bytes = GR * (int)sizeof(T), piece = bytes >= 16 ? 16 : 4, per = bytes / piece;
  static_assert(bytes % 4 == 0, "cp.async moves 4 or 16 bytes");
#pragma unroll
  for (int n = 0; n < CH * 8 / GR; ++n) {
    const int j = (n * G + t) * GR;
    if (j < d) {
#pragma unroll
      for (int i = 0; i < per; ++i) {
        const uint32_t dst = (uint32_t)__cvta_generic_to_shared(slot + (((n * per + i) * G + t) * piece));
        const char* src = (const char*)(row + j) + i * piece;
        if (piece == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
      }
    }
  }
}
template <int GR, typename T>
__device__ __forceinline__ void read_slot(float (&o)[8], const char* slot, int c, int t, int G, int d) {
  constexpr int bytes = GR * (int)sizeof(T), piece = bytes >= 16 ? 16 : 4, per = bytes / piece;
  Raw8<T> r;
#pragma unroll
  for (int n = 0; n < 8 / GR; ++n)
#pragma unroll
    for (int i = 0; i < per; ++i) {
      const char* src = slot + (((c * (8 / GR) + n) * per + i) * G + t) * piece;
      if (piece == 16) ((uint4*)r.v)[n * per + i] = *(const uint4*)src;
      else ((uint32_t*)r.v)[n * per + i] = *(const uint32_t*)src;
    }
#pragma unroll
  for (int k = 0; k < 8; ++k) o[k] = column<GR>(c, k, t, G) < d ? to_f(r.v[k]) : 0.f;
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// until at most `later` of this thread's groups are still in flight
__device__ __forceinline__ void copies_wait(int later) {
  if (later <= 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else if (later == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else asm volatile("cp.async.wait_group 3;" ::: "memory");
}
static constexpr int MAX_AHEAD = 3;

// Sums of NV values over the G threads of a row, every thread receiving the same bits.  A butterfly within each warp,
// then (G > 32) the warps' sums through shared memory and a second butterfly.  `red` has two halves used in turn, so
// one block barrier per call is enough.
static constexpr int RED_VALUES = 3;
template <int NV>
__device__ __forceinline__ void row_sums(float (&v)[NV], float* red, int& half, int G, int t) {
#pragma unroll
  for (int o = 16; o; o >>= 1)
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  if (G > 32) {
    float* r = red + half * (RED_VALUES * 16);
    half ^= 1;
    const int warps = G >> 5;
    if ((t & 31) == 0)
#pragma unroll
      for (int i = 0; i < NV; ++i) r[i * 16 + (t >> 5)] = v[i];
    __syncthreads();
    // every half warp adds the (at most 16) warps' sums
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = (t & 15) < warps ? r[i * 16 + (t & 15)] : 0.f;
#pragma unroll
    for (int o = 8; o; o >>= 1)
#pragma unroll
      for (int i = 0; i < NV; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  }
}

__device__ __forceinline__ float sigmoid_f(float v) { return __fdividef(1.f, 1.f + __expf(-v)); }

struct Args {
  int64_t rows;
  int d, G;
  int ahead;                // rows fetched ahead of the present one, 1 .. MAX_AHEAD (kernels that fetch ahead)
  int slot_bytes;           // of one row, all streams
  int pre, post, gate, bias;
  unsigned per_gate;
  float eps, inv_d;
  const float* params;      // [w_pre, w_post, s (, b_pre, b_post)], d values each
  const void* x; int64_t ldx;          // forward: x; backward: x'
  const void* y; int64_t ldy;          // may be null
  const void* g; int64_t ldg;
  void* x_out; int64_t ldxo;           // forward
  void* u; int64_t ldu;                // forward, may be null
  const void* du; int64_t lddu;        // backward, may be null
  const void* dxo; int64_t lddxo;      // backward, may be null
  void* dx; int64_t lddx;
  void* dy; int64_t lddy;
  void* dg; int64_t lddg;
  float* gate_partials;                // [walkers + gates, d] (gates of several rows)
  float* col_partials;                 // [blocks, quantities, d]
  int walkers;                         // row-holding thread groups of the whole grid
};

// How a call's rows are laid over threads.
struct Layout {
  int granule;              // 8, 2 or 1
  int G, chunks;            // threads per row, chunks of 8 values per thread
  int threads;              // of a block
  int blocks_per_sm;        // that the grid counts on
  int ahead, slot_bytes;    // ahead 0: rows are read from global memory where they are used
  size_t smem;
};

// streams of the residual stream's type and of the block's type that a row fetches; threads_per_sm: what the kernel's
// registers allow; chunks: values per thread / 8 to aim for where rows are aligned
Layout layout_of(int64_t d, int x_dtype, int y_dtype, int granule, int streams_x, int streams_y, int threads_per_sm, int chunks);
betty_status forward(cudaStream_t stream, Args& a, int x_dtype, int y_dtype, int granule);
Layout backward_layout(int64_t d, int x_dtype, int y_dtype, int granule);
int backward_blocks(int64_t rows, const Layout& l);
betty_status backward(cudaStream_t stream, Args& a, const Layout& l, int x_dtype, int y_dtype, float* dparams);

}  // namespace blocknorm
}  // namespace betty
