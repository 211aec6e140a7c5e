// Norms before and after a residual block, fused with its gate and residual scale.
//
//   m = N_post(y)      z = m * w_post (+ b_post)      x' = x + s * a(g) * z      u = N_pre(x') * w_pre (+ b_pre)
//
// N is the identity, the RMS norm  v / sqrt(mean(v^2) + eps)  or the layer norm (the same of v - mean(v)); a is 1, the
// gate itself or its sigmoid.  The shared pieces of the forward and the backward kernel: how a row is laid over
// threads, how rows are fetched ahead, and the sums over a row.
#pragma once
#include "values.cuh"

namespace betty {
namespace blocknorm {

// A row is held by G threads (a multiple of 32 up to MAX_G; a block's eight warps hold eight rows where G is 32, otherwise
// a block holds one), CH * 8 values each.  VEC: chunk c of thread t is the eight values from (c * G + t) * 8 - shift, one or
// two 16-byte accesses, where shift is how far the row starts behind a 16-byte boundary (counted modulo 8 values).  Rows of an odd width start at every shift in turn; the rows that one thread group
// takes all have the same one ("class": rows of equal number modulo `classes`), so that a thread's columns, and with them
// its parameters and column sums, stay the same.  Otherwise (matrices whose rows start at different shifts, or wider rows
// than shared memory holds) values are accessed one by one: value k of chunk c is column (c * 8 + k) * G + t.
static constexpr int MAX_G = 512;
static constexpr int MAX_CH = 4;
static constexpr int MAX_D = MAX_G * 8 * MAX_CH;
static constexpr int SMALL_THREADS = 256;     // block size when a warp holds a row

// where a thread's values lie in a row
struct Place { int t, G, d, shift; };
template <bool VEC>
__device__ __forceinline__ int column(const Place& w, int c, int k) {
  return VEC ? (c * w.G + w.t) * 8 + k - w.shift : (c * 8 + k) * w.G + w.t;
}
template <bool VEC>
__device__ __forceinline__ bool inside(const Place& w, int c, int k) { return (unsigned)column<VEC>(w, c, k) < (unsigned)w.d; }

// chunk c of a row in global memory, value by value; columns outside the row are 0
template <bool VEC, typename T>
__device__ __forceinline__ void load8(float (&o)[8], const T* row, int c, const Place& w) {
#pragma unroll
  for (int k = 0; k < 8; ++k) o[k] = inside<VEC>(w, c, k) ? to_f(row[column<VEC>(w, c, k)]) : 0.f;
}
template <bool VEC, typename T>
__device__ __forceinline__ void store_each(T* row, const float (&v)[8], int c, const Place& w) {
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (inside<VEC>(w, c, k)) row[column<VEC>(w, c, k)] = from_f<T>(v[k]);
}
// rows of the call's matrices: 16 bytes at a time except at a shifted row's ends
template <bool VEC, typename T>
__device__ __forceinline__ void store8(T* row, const float (&v)[8], int c, const Place& w) {
  if constexpr (VEC) {
    const int j = column<VEC>(w, c, 0);
    if (j >= 0 && j + 8 <= w.d) {
      if constexpr (sizeof(T) == 4) {
        *(float4*)(row + j) = make_float4(v[0], v[1], v[2], v[3]);
        *(float4*)(row + j + 4) = make_float4(v[4], v[5], v[6], v[7]);
      } else {
        *(uint4*)(row + j) = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
      }
      return;
    }
    if (j >= w.d) return;
  }
  store_each<VEC>(row, v, c, w);
}

// ---- shared memory by 32-bit addresses: half the registers of generic pointers ----
__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ float4 lds16f(uint32_t a) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ void sts16f(uint32_t a, float x, float y, float z, float w) {
  asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(a), "f"(x), "f"(y), "f"(z), "f"(w) : "memory");
}
__device__ __forceinline__ float lds4f(uint32_t a) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ void sts4f(uint32_t a, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(a), "f"(v) : "memory"); }
template <typename T> __device__ __forceinline__ void sts(uint32_t a, T v) {
  if constexpr (sizeof(T) == 4) sts4f(a, v);
  else asm volatile("st.shared.b16 [%0], %1;" ::"r"(a), "h"(*(const uint16_t*)&v) : "memory");
}

// ---- rows fetched ahead ----
// Each thread copies the 16-byte pieces that it will itself read into its own slots of shared memory with cp.async, a few
// rows before their use: no registers are held by data in flight, and as nobody reads another thread's slots, waiting for
// one's own copies is all the synchronisation there is.  A slot holds CH * 8 values of every stream, interleaved over the
// G threads so that a warp's accesses are contiguous.  Columns from d on are filled with zeros (a copy of fewer bytes); the
// values before column 0 of a shifted row are the end of the row before (never before the matrix: its first row has shift
// 0) and are cleared by drop_head.
template <int CH, typename T>
__device__ __forceinline__ void copy_row(uint32_t slot, const T* row, const Place& w) {
  constexpr int per = (int)sizeof(T) / 2, values = 16 / (int)sizeof(T);
  const uint32_t dst = slot + w.t * 16;
  const T* base = row - w.shift;
  if (w.d == CH * 8 * w.G) {         // nothing to fill (and no shift: the threads then hold seven columns more than d)
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < per; ++i)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                     ::"r"(dst + (c * per + i) * w.G * 16), "l"(base + (c * w.G + w.t) * 8 + i * values) : "memory");
    return;
  }
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < per; ++i) {
      const int j = (c * w.G + w.t) * 8 + i * values, left = (w.d + w.shift - j) * (int)sizeof(T), size = left < 0 ? 0 : (left > 16 ? 16 : left);
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                   ::"r"(dst + (c * per + i) * w.G * 16), "l"(size > 0 ? base + j : base), "r"(size) : "memory");
    }
}
// the same for a row at another shift than the thread's columns, value by value and not ahead
template <int CH, bool VEC, typename T>
__device__ __forceinline__ void fill_slot(uint32_t slot, const T* row, const Place& w) {
#pragma unroll 1
  for (int c = 0; c < CH; ++c)
#pragma unroll 1
    for (int k = 0; k < 8; ++k)
      sts<T>(slot + ((c * (int)sizeof(T) / 2 + k * (int)sizeof(T) / 16) * w.G + w.t) * 16 + k * (int)sizeof(T) % 16,
             inside<VEC>(w, c, k) ? row[column<VEC>(w, c, k)] : from_f<T>(0.f));
}
template <typename T>
__device__ __forceinline__ void drop_head(uint32_t slot, const Place& w) {
  if (w.t == 0)
    for (int k = 0; k < w.shift; ++k) sts<T>(slot + (k * (int)sizeof(T) / 16) * w.G * 16 + k * (int)sizeof(T) % 16, from_f<T>(0.f));
}
template <typename T>
__device__ __forceinline__ void read_slot(float (&o)[8], uint32_t slot, int c, const Place& w) {
  if constexpr (sizeof(T) == 4) {
    const float4 a = lds16f(slot + ((c * 2) * w.G + w.t) * 16), b = lds16f(slot + ((c * 2 + 1) * w.G + w.t) * 16);
    o[0] = a.x; o[1] = a.y; o[2] = a.z; o[3] = a.w; o[4] = b.x; o[5] = b.y; o[6] = b.z; o[7] = b.w;
  } else {
    const uint4 a = lds16(slot + (c * w.G + w.t) * 16);
    unpack2<T>(a.x, o[0], o[1]); unpack2<T>(a.y, o[2], o[3]); unpack2<T>(a.z, o[4], o[5]); unpack2<T>(a.w, o[6], o[7]);
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
// P - 1 exchanges and log2(32 / P) further ones instead of 5 P.  Across warps every thread then adds the warps' sums from
// shared memory (broadcast reads).  `red` has two halves used in turn, so one block barrier per call is enough.
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
  const int warps = G >> 5;
  if (lane % (32 / P) == 0) r[lane / (32 / P) * 16 + (t >> 5)] = u[0];
  __syncthreads();
  // every thread adds them in the same order, four at a time (the places of absent warps hold zeros)
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const float4 w = *(const float4*)(r + i * 16);
    v[i] = (w.x + w.y) + (w.z + w.w);
  }
  for (int j = 4; j < warps; j += 4) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const float4 w = *(const float4*)(r + i * 16 + j);
      v[i] += (w.x + w.y) + (w.z + w.w);
    }
  }
}
// once, before the first sum
__device__ __forceinline__ void row_sums_init(float* red) {
  for (int i = threadIdx.x; i < 2 * RED_VALUES * 16; i += blockDim.x) red[i] = 0.f;
  __syncthreads();
}

// A sigmoid gate and 1 - it.  A residual stream in fp32 takes them to 7e-7 of themselves; where all results are rounded to 16 bits the
// fast forms do, 2^-22 (2 + |v|) of the gate (for its complement, of 1).
template <typename TX>
__device__ __forceinline__ void sigmoid_gate(float v, float& s, float& n) {
  if constexpr (sizeof(TX) == 4) {
    sigmoid_parts(v, s, n);
  } else {
    s = __fdividef(1.f, 1.f + __expf(-v));
    n = 1.f - s;
  }
}
template <typename TX>
__device__ __forceinline__ float sigmoid_gate(float v) {
  float s, n;
  sigmoid_gate<TX>(v, s, n);
  return s;
}

// places of the walkers' sums for gates of several rows (see gate_slot)
struct GateSums { int64_t rows; unsigned per_share, per_gate, per_row, begins; };

struct Args {
  int64_t rows;
  int d, G;
  int classes;              // 1, 2, 4 or 8: row r starts at the shift of row r % classes,
  int ld8;                  // which is (r * ld8) modulo 8
  int ahead;                // batches of rows fetched ahead of the present one, up to MAX_AHEAD (kernels that fetch ahead)
  int slot_bytes;           // of one row, all streams
  int pre, post, gate, bias;
  unsigned per_gate;
  int gate_ahead;           // forward: the gate is among the streams fetched ahead
  float eps, inv_d;
  const float* params;      // [w_pre, w_post, s (, b_pre, b_post)], d values each
  // matrices: address and bytes from one row to the next
  const void* x; uint32_t ldx;          // forward: x; backward: x'
  const void* y; uint32_t ldy;          // may be null
  const void* g; uint32_t ldg;
  void* x_out; uint32_t ldxo;           // forward
  void* u; uint32_t ldu;                // forward, may be null
  const void* du; uint32_t lddu;        // backward, may be null
  const void* dxo; uint32_t lddxo;      // backward, may be null
  void* dx; uint32_t lddx;
  void* dy; uint32_t lddy;
  void* dg; uint32_t lddg;
  float* gate_partials;                // [classes][gate_sums.rows][d] (gates of several rows)
  GateSums gate_sums;
  float* col_partials;                 // [blocks, quantities, d]
  int shares;                          // backward: contiguous shares that the rows of a class are cut into
};

// How a call's rows are laid over threads.
struct Layout {
  bool vec;
  int G, chunks;            // threads per row, chunks of 8 values per thread
  int threads;              // of a block
  int blocks_per_sm;        // that the grid counts on
  bool wide;                // two chunks and several rows at a time: many rows; else the shortest way for a few
  int ahead, slot_bytes;    // batches fetched ahead; 0 with vec: a row is fetched when it is its turn
  size_t smem;
};

struct Needs {
  int streams_x, streams_y; // rows fetched of the residual stream's and of the block's type
  int wide_chunks, batch;   // of the wide kernel
  int kept_arrays;          // fp32 values of a row that each thread group keeps in shared memory beside fetched rows (coefficients)
  int sum_arrays;           // and beside any rows (sums)
};
// classes: 0 where the matrices' rows do not start at one shift
Layout layout_of(int64_t d, int64_t rows, int x_dtype, int y_dtype, int classes, const Needs& n);
betty_status forward(cudaStream_t stream, Args& a, int x_dtype, int y_dtype, int classes);
Layout backward_layout(const betty_block_norm_cfg* c, int64_t rows, int x_dtype, int y_dtype, int classes);
void backward_grid(int64_t rows, const Layout& l, int classes, int& blocks, int& shares);
GateSums gate_sums_of(int64_t rows, int64_t per_gate, int classes, int shares);
betty_status backward(cudaStream_t stream, Args& a, const Layout& l, int x_dtype, int y_dtype, float* dparams);

}  // namespace blocknorm
}  // namespace betty
