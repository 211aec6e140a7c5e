// Norms before and after a residual block, fused with its gate and residual scale.
//
//   m = N_post(y)      z = m * w_post (+ b_post)      x' = x + s * a(g) * z      u = N_pre(x') * w_pre (+ b_pre)
//
// N is the identity, the RMS norm  v / sqrt(mean(v^2) + eps)  or the layer norm (the same of v - mean(v)); a is 1, the
// gate itself or its sigmoid.  The shared pieces of the forward and the backward kernel: how a row is laid over
// threads, loads and stores, and the sums over a row.
#pragma once
#include "common.cuh"

namespace betty {
namespace blocknorm {

// A row is held by G threads (a power of two, 32 .. MAX_G), CH * 8 values each.  Aligned rows: chunk c of thread t is
// the 8 consecutive values from (c * G + t) * 8, one or two 16-byte accesses.  Other rows (odd widths, odd strides):
// the same 8 registers hold values c * 8G + k * G + t, so that the threads of a warp touch neighbours.
static constexpr int MAX_G = 512;
static constexpr int MAX_D = MAX_G * 8 * 4;
static constexpr int SMALL_THREADS = 256;     // block size when a warp holds a row

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f(float v) { return v; }
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f(float v) { return __float2half_rn(v); }

template <bool ALIGNED>
__device__ __forceinline__ int column(int c, int k, int t, int G) {
  return ALIGNED ? (c * G + t) * 8 + k : (c * 8 + k) * G + t;
}

// Eight values as they lie in memory, so that a row requested ahead of its use costs no more registers than its bytes.
template <typename T> struct alignas(16) Raw8 { T v[8]; };

template <bool ALIGNED, typename T>
__device__ __forceinline__ void load8(Raw8<T>& r, const T* row, int c, int t, int G, int d) {
  if (ALIGNED) {
    const int j = (c * G + t) * 8;
    if (j < d) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) ((uint4*)r.v)[i] = *(const uint4*)((const char*)(row + j) + 16 * i);
    } else {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) ((uint4*)r.v)[i] = make_uint4(0, 0, 0, 0);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int j = (c * 8 + k) * G + t;
      r.v[k] = j < d ? row[j] : from_f<T>(0.f);
    }
  }
}
template <bool ALIGNED, typename T>
__device__ __forceinline__ void store8(T* row, const float (&v)[8], int c, int t, int G, int d) {
  if (ALIGNED) {
    const int j = (c * G + t) * 8;
    if (j < d) {
      Raw8<T> r;
#pragma unroll
      for (int k = 0; k < 8; ++k) r.v[k] = from_f<T>(v[k]);
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) *(uint4*)((char*)(row + j) + 16 * i) = ((const uint4*)r.v)[i];
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int j = (c * 8 + k) * G + t;
      if (j < d) row[j] = from_f<T>(v[k]);
    }
  }
}
// parameters are fp32; values beyond d read as `pad`
template <bool ALIGNED>
__device__ __forceinline__ void load_param8(float (&v)[8], const float* row, int c, int t, int G, int d) {
  if (ALIGNED) {
    const int j = (c * G + t) * 8;
    if (j < d) {
      const float4 a = *(const float4*)(row + j), b = *(const float4*)(row + j + 4);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = 0.f;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int j = (c * 8 + k) * G + t;
      v[k] = j < d ? row[j] : 0.f;
    }
  }
}

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
    float* r = red + half * (RED_VALUES * 32);
    half ^= 1;
    const int warps = G >> 5;
    if ((t & 31) == 0)
#pragma unroll
      for (int i = 0; i < NV; ++i) r[i * 32 + (t >> 5)] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = (t & 31) < warps ? r[i * 32 + (t & 31)] : 0.f;
    for (int o = warps >> 1; o; o >>= 1)
#pragma unroll
      for (int i = 0; i < NV; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = __shfl_sync(0xffffffffu, v[i], 0);
  }
}

__device__ __forceinline__ float sigmoid_f(float v) { return __fdividef(1.f, 1.f + __expf(-v)); }

struct Args {
  int64_t rows;
  int d, G;
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

// threads that hold a row of d values, and chunks of 8 each holds
static inline int threads_per_row(int64_t d) {
  int G = 32;
  while (G < MAX_G && (int64_t)G * 8 < d) G *= 2;
  return G;
}
static inline int chunks_of(int64_t d, int G) { return (int)((d + (int64_t)G * 8 - 1) / ((int64_t)G * 8)); }

betty_status forward(cudaStream_t stream, const Args& a, int x_dtype, int y_dtype, bool aligned);
betty_status backward(cudaStream_t stream, Args& a, int x_dtype, int y_dtype, bool aligned, float* dparams);
int backward_blocks(int64_t rows, int G);

}  // namespace blocknorm
}  // namespace betty
