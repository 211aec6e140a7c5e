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

// two neighbouring values into one 32-bit word, one conversion instruction
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *(const uint32_t*)&v;
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *(const uint32_t*)&v;
}
template <typename T> __device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b);
template <> __device__ __forceinline__ void unpack2<__nv_bfloat16>(uint32_t w, float& a, float& b) {
  a = __uint_as_float(w << 16);
  b = __uint_as_float(w & 0xffff0000u);
}
template <> __device__ __forceinline__ void unpack2<__half>(uint32_t w, float& a, float& b) {
  const float2 v = __half22float2(*(const __half2*)&w);
  a = v.x; b = v.y;
}

// column of a thread's value k (0 .. 7) of chunk c
template <int GR>
__device__ __forceinline__ int column(int c, int k, int t, int G) {
  return ((c * (8 / GR) + k / GR) * G + t) * GR + k % GR;
}

// chunk c of a row in global memory; columns beyond d are 0
template <int GR, typename T>
__device__ __forceinline__ void load8(float (&o)[8], const T* row, int c, int t, int G, int d) {
  if constexpr (GR == 8) {
    const int j = (c * G + t) * 8;
    uint4 w[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = j < d ? *(const uint4*)((const char*)(row + j) + 16 * i) : make_uint4(0, 0, 0, 0);
    if constexpr (sizeof(T) == 4) {
      o[0] = __uint_as_float(w[0].x); o[1] = __uint_as_float(w[0].y); o[2] = __uint_as_float(w[0].z); o[3] = __uint_as_float(w[0].w);
      o[4] = __uint_as_float(w[1].x); o[5] = __uint_as_float(w[1].y); o[6] = __uint_as_float(w[1].z); o[7] = __uint_as_float(w[1].w);
    } else {
      unpack2<T>(w[0].x, o[0], o[1]); unpack2<T>(w[0].y, o[2], o[3]); unpack2<T>(w[0].z, o[4], o[5]); unpack2<T>(w[0].w, o[6], o[7]);
    }
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
  if constexpr (GR == 8) {
    const int j = (c * G + t) * 8;
    if (j < d) {
      if constexpr (sizeof(T) == 4) {
        *(float4*)(row + j) = make_float4(v[0], v[1], v[2], v[3]);
        *(float4*)(row + j + 4) = make_float4(v[4], v[5], v[6], v[7]);
      } else {
        *(uint4*)(row + j) = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
      }
    }
  } else if constexpr (GR == 2 && sizeof(T) == 2) {
#pragma unroll
    for (int k = 0; k < 8; k += 2) {             // rows start on 4-byte boundaries and d is even
      const int j = column<GR>(c, k, t, G);
      if (j < d) *(uint32_t*)(row + j) = pack2<T>(v[k], v[k + 1]);
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
// Columns beyond d are filled with zeros (a copy of no bytes), so that reading a slot needs no comparison.
template <int GR, int CH, typename T>
__device__ __forceinline__ void copy_row(char* slot, const T* row, int t, int G, int d) {
  constexpr int bytes = GR * (int)sizeof(T), piece = bytes >= 16 ? 16 : 4, per = bytes / piece;
  static_assert(bytes % 4 == 0, "cp.async moves 4 or 16 bytes");
  const uint32_t dst = (uint32_t)__cvta_generic_to_shared(slot) + t * piece;
#pragma unroll
  for (int n = 0; n < CH * 8 / GR; ++n) {
    const int j = (n * G + t) * GR, size = j < d ? piece : 0;
    const char* src = (const char*)(row + (j < d ? j : 0));
#pragma unroll
    for (int i = 0; i < per; ++i) {
      if (piece == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + (n * per + i) * G * piece), "l"(src + i * piece), "r"(size) : "memory");
      else
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst + (n * per + i) * G * piece), "l"(src + i * piece), "r"(size) : "memory");
    }
  }
}
template <int GR, typename T>
__device__ __forceinline__ void read_slot(float (&o)[8], const char* slot, int c, int t, int G) {
  constexpr int bytes = GR * (int)sizeof(T), piece = bytes >= 16 ? 16 : 4, pieces = 8 * (int)sizeof(T) / piece;
#pragma unroll
  for (int i = 0; i < pieces; ++i) {
    const char* src = slot + ((c * pieces + i) * G + t) * piece;
    constexpr int per = piece / (int)sizeof(T);          // values in a piece
    if constexpr (piece == 16 && sizeof(T) == 4) {
      const float4 w = *(const float4*)src;
      o[i * per] = w.x; o[i * per + 1] = w.y; o[i * per + 2] = w.z; o[i * per + 3] = w.w;
    } else if constexpr (piece == 16) {
      const uint4 w = *(const uint4*)src;
      unpack2<T>(w.x, o[0], o[1]); unpack2<T>(w.y, o[2], o[3]); unpack2<T>(w.z, o[4], o[5]); unpack2<T>(w.w, o[6], o[7]);
    } else if constexpr (sizeof(T) == 4) {
      o[i] = *(const float*)src;
    } else {
      unpack2<T>(*(const uint32_t*)src, o[2 * i], o[2 * i + 1]);
    }
  }
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// until at most `later` of this thread's groups are still in flight
__device__ __forceinline__ void copies_wait(int later) {
  if (later <= 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else if (later == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else asm volatile("cp.async.wait_group 3;" ::: "memory");
}
static constexpr int MAX_AHEAD = 3;

// Sums of NV values over the G threads of a row, every thread receiving the same bits.  Within a warp the values are
// folded while they are reduced: each of the first steps halves the number of values a lane carries, so that P values cost
// P - 1 exchanges and log2(32 / P) further ones instead of 5 P.  Across warps every lane then takes one (value, warp) pair
// from shared memory.  `red` has two halves used in turn, so one block barrier per call is enough.
static constexpr int RED_VALUES = 8;
template <int NV>
__device__ __forceinline__ void row_sums(float (&v)[NV], float* red, int& half, int G, int t) {
  constexpr int P = NV <= 1 ? 1 : (NV <= 2 ? 2 : (NV <= 4 ? 4 : 8));
  const int lane = t & 31;
  float u[P];
#pragma unroll
  for (int i = 0; i < P; ++i) u[i] = i < NV ? v[i < NV ? i : 0] : 0.f;
#pragma unroll
  for (int n = P, o = 16; o; o >>= 1) {
    if (n > 1) {
      n >>= 1;
      const bool up = lane & o;
#pragma unroll
      for (int i = 0; i < n; ++i) {
        const float send = up ? u[i] : u[i + n], keep = up ? u[i + n] : u[i];
        u[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
      }
    } else {
      u[0] += __shfl_xor_sync(0xffffffffu, u[0], o);
    }
  }
  if (G == 32) {           // value i now is in lanes i * 32 / P ...
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = P == 1 ? u[0] : __shfl_sync(0xffffffffu, u[0], i * (32 / P));
    return;
  }
  float* r = red + half * (RED_VALUES * 16);
  half ^= 1;
  const int warps = G >> 5, lg = 31 - __clz(warps);
  if (lane % (32 / P) == 0) r[((lane / (32 / P)) << lg) + (t >> 5)] = u[0];
  __syncthreads();
  constexpr int LOADS = P * 16 > 32 ? P * 16 / 32 : 1;       // at most 16 warps
  float w[LOADS];
#pragma unroll
  for (int j = 0; j < LOADS; ++j) {
    const int e = lane + 32 * j;
    w[j] = r[e & ((P << lg) - 1)];
  }
#pragma unroll
  for (int o = 8; o; o >>= 1)
    if (o < warps)
#pragma unroll
      for (int j = 0; j < LOADS; ++j) w[j] += __shfl_xor_sync(0xffffffffu, w[j], o);
#pragma unroll
  for (int i = 0; i < NV; ++i) {                              // pair e = i * warps + ... is in lane e % 32 of load e / 32
    const int e = i << lg;
    float x = w[0];
#pragma unroll
    for (int j = 1; j < LOADS; ++j)
      if ((e >> 5) == j) x = w[j];
    v[i] = __shfl_sync(0xffffffffu, x, e & 31);
  }
}

// ---- pairs of fp32 values: one instruction for two products or sums ----
struct alignas(8) f2 { float x, y; };
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 r;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 r;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 r;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ f2 both(float v) { return f2{v, v}; }
__device__ __forceinline__ void pairs(f2 (&o)[4], const float (&v)[8]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] = f2{v[2 * k], v[2 * k + 1]};
}
__device__ __forceinline__ void singles(float (&o)[8], const f2 (&v)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) { o[2 * k] = v[k].x; o[2 * k + 1] = v[k].y; }
}

__device__ __forceinline__ float sigmoid_f(float v) { return __fdividef(1.f, 1.f + __expf(-v)); }

struct Args {
  int64_t rows;
  int d, G;
  int ahead;                // batches of rows fetched ahead of the present one, 1 .. MAX_AHEAD (kernels that fetch ahead)
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
  int walkers;                         // thread groups with rows, at most one per row
};

// How a call's rows are laid over threads.
struct Layout {
  int granule;              // 8, 2 or 1
  int G, chunks;            // threads per row, chunks of 8 values per thread
  int threads;              // of a block
  int blocks_per_sm;        // that the grid counts on
  bool wide;                // two chunks and several rows at a time: many rows; else the shortest way for a few
  int ahead, slot_bytes;    // batches fetched ahead; 0: rows are read from global memory where they are used
  size_t smem;
};

struct Needs {
  int streams_x, streams_y; // rows fetched of the residual stream's and of the block's type
  int wide_chunks, batch;   // of the wide kernel
  int acc_arrays;           // fp32 values of a row that each thread group keeps in shared memory
  int param_arrays;         // and that a block keeps once
};
Layout layout_of(int64_t d, int64_t rows, int x_dtype, int y_dtype, int granule, const Needs& n);
betty_status forward(cudaStream_t stream, Args& a, int x_dtype, int y_dtype, int granule);
Layout backward_layout(const betty_block_norm_cfg* c, int64_t rows, int x_dtype, int y_dtype, int granule);
int backward_blocks(int64_t rows, const Layout& l);
betty_status backward(cudaStream_t stream, Args& a, const Layout& l, int x_dtype, int y_dtype, float* dparams);

}  // namespace blocknorm
}  // namespace betty
