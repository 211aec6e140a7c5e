// 8-bit checkpoints of a hidden layer's pre-activations, and the layer's backward pass from them.
//
// A row of z (or each half of a gated row [gate | value]) is cut into groups of 128 values.  A group is held as whole
// numbers in [-127, 127] and one fp32 scale:
//
//   top = max |z|,   q = rint(z * (127 * (1 / top))),   scale = top * (1 / 127),   z~ = q * scale
//
// every operation rounded to fp32 on its own (no contraction), so that q is the same whoever computes it.  A group whose
// top is below 1e-30 is held as zeros; one that holds an infinity or a NaN gets the scale NaN, so that it stays visible.
//
//   store:     a = act(z)                 or  act(z_gate) * z_value;  z -> q, scale
//   backward:  dz = da * act'(z~)         or  [da * z~_value * act'(z~_gate) | da * act(z~_gate)];   a from z~ for the
//              weight gradient of the next layer, which so needs no stored activation either
//
// All three kernels are bound by memory (5 to 7 bytes per value at ~30 operations, 2 of them on the special-function
// pipe): rounding and the bytes' conversion go through additions of 1.5 * 2^23 and byte permutes, not through the
// conversion instructions, which share that pipe with exp and the reciprocal.
#include "gemm.cuh"

namespace betty {
namespace act8 {

static constexpr int GROUP = 128;
static constexpr int LANES = 16;              // half a warp holds a group, 8 values per lane
static constexpr int THREADS = 256;
static constexpr int UNITS = THREADS / LANES; // groups a block holds at a time
static constexpr float TINY = 1e-30f;

struct Args {
  int64_t rows;
  int cols, groups;        // per part
  int unit_cols;           // groups of one row a block holds side by side (a power of two), UNITS / unit_cols rows deep
  const void* z; int64_t ldz;
  void* a; int64_t lda;
  int8_t* q; int64_t ldq;
  float* scales; int64_t lds;
  const void* da; int64_t ldda;
  void* dz; int64_t lddz;
};

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f(float v) { return v; }
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f(float v) { return __float2half_rn(v); }

template <typename T> struct alignas(16) Raw8 { T v[8]; };

// Lane l of a group's half warp holds its values 8l .. 8l+7 where rows allow 16-byte accesses, else l, l+16, ...
template <bool ALIGNED> __device__ __forceinline__ int place(int lane, int k) { return ALIGNED ? lane * 8 + k : lane + k * LANES; }

// v[k] = row[at + place] for the places below n, else 0
template <bool ALIGNED, typename T>
__device__ __forceinline__ void load8(float (&v)[8], const T* row, int lane, int n) {
  Raw8<T> r;
  if (ALIGNED) {
    if (lane * 8 < n) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) ((uint4*)r.v)[i] = *(const uint4*)((const char*)(row + lane * 8) + 16 * i);
    } else {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) ((uint4*)r.v)[i] = make_uint4(0, 0, 0, 0);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) r.v[k] = lane + k * LANES < n ? row[lane + k * LANES] : from_f<T>(0.f);
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = to_f(r.v[k]);
}
template <bool ALIGNED, typename T>
__device__ __forceinline__ void store8(T* row, const float (&v)[8], int lane, int n) {
  if (ALIGNED) {
    if (lane * 8 < n) {
      Raw8<T> r;
#pragma unroll
      for (int k = 0; k < 8; ++k) r.v[k] = from_f<T>(v[k]);
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) *(uint4*)((char*)(row + lane * 8) + 16 * i) = ((const uint4*)r.v)[i];
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (lane + k * LANES < n) row[lane + k * LANES] = from_f<T>(v[k]);
  }
}

// z -> q (its fp32 holder's low byte) and the group's scale
template <bool ALIGNED>
__device__ __forceinline__ void quantise(const float (&z)[8], int8_t* q, float* scale, int lane, int n) {
  uint32_t top = 0;                     // largest magnitude by its bits: orders finite < infinity < NaN
#pragma unroll
  for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint(z[k]) & 0x7fffffffu);
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  const float t = __uint_as_float(top);
  const bool bad = top >= 0x7f800000u, some = t >= TINY && !bad;
  const float inv = some ? __fmul_rn(__frcp_rn(t), 127.f) : 0.f;
  uint32_t b[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) b[k] = some ? __float_as_uint(__fadd_rn(__fmul_rn(z[k], inv), 12582912.f)) : 0u;
  if (ALIGNED) {
    if (lane * 8 < n) {
      uint2 w;
      w.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
      w.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
      *(uint2*)(q + lane * 8) = w;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (lane + k * LANES < n) q[lane + k * LANES] = (int8_t)(b[k] & 0xffu);
  }
  if (lane == 0) *scale = bad ? __uint_as_float(0x7fffffffu) : (some ? __fmul_rn(t, 1.f / 127.f) : 0.f);
}
template <bool ALIGNED>
__device__ __forceinline__ void restore(float (&z)[8], const int8_t* q, float scale, int lane, int n) {
  uint32_t w[2] = {0, 0};
  if (ALIGNED) {
    if (lane * 8 < n) { const uint2 v = *(const uint2*)(q + lane * 8); w[0] = v.x; w[1] = v.y; }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (lane + k * LANES < n) w[k >> 2] |= (uint32_t)(uint8_t)q[lane + k * LANES] << (8 * (k & 3));
  }
  w[0] ^= 0x80808080u; w[1] ^= 0x80808080u;          // q + 128, a byte that becomes the low bits of 2^23 + q + 128
#pragma unroll
  for (int k = 0; k < 8; ++k)
    z[k] = __fmul_rn(__uint_as_float(__byte_perm(w[k >> 2], 0x4b000000u, 0x7650 + (k & 3))) - 8388736.f, scale);
}

// Activation and its slope.  16-bit results take the distribution function of gemm.cuh (|error| <= 1.5e-7); fp32 ones erff.
template <typename T, int ACT>
__device__ __forceinline__ void act_and_slope(float v, float& f, float& s) {
  if (ACT == BETTY_ACT_RELU) {
    f = fmaxf(v, 0.f);
    s = v > 0.f ? 1.f : 0.f;
    if (v != v) { f = v; s = v; }
  } else if (ACT == BETTY_ACT_SILU) {
    const float e = __fdividef(1.f, 1.f + __expf(-v));
    f = v * e;
    s = e * fmaf(v, 1.f - e, 1.f);
  } else {
    const float c = sizeof(T) == 4 ? 0.5f * (1.f + erff(v * 0.7071067811865476f)) : fam_bf16::norm_cdf(v);
    f = v * c;
    s = fmaf(v, fam_bf16::norm_pdf(v), c);
  }
}

struct Walk { int lane, group, at, n; int64_t row, step; };
__device__ __forceinline__ Walk walk(const Args& a) {
  Walk w;
  const int unit = threadIdx.x / LANES, deep = UNITS / a.unit_cols;
  w.lane = threadIdx.x & (LANES - 1);
  w.group = blockIdx.x * a.unit_cols + (unit & (a.unit_cols - 1));
  w.at = w.group * GROUP;
  w.n = min(GROUP, a.cols - w.at);                   // <= 0: this unit has no group; it still takes part in the shuffles
  w.row = (int64_t)blockIdx.y * deep + unit / a.unit_cols;
  w.step = (int64_t)gridDim.y * deep;
  return w;
}
// rows are walked by whole warps (two units): a unit past the last row masks its accesses but stays in the shuffles
__device__ __forceinline__ bool warp_has_rows(const Walk& w, int64_t rows) { return __any_sync(0xffffffffu, w.row < rows && w.n > 0); }

template <typename T, int ACT, bool GATED, bool ALIGNED>
__global__ void __launch_bounds__(THREADS) k_store(const Args a) {
  pdl_enter();
  Walk w = walk(a);
  for (; warp_has_rows(w, a.rows); w.row += w.step) {
    const int n = w.row < a.rows ? w.n : 0;
    const int64_t row = n > 0 ? w.row : 0;
    const T* z = (const T*)a.z + row * a.ldz + w.at;
    float g[8], v[8];
    load8<ALIGNED>(g, z, w.lane, n);
    if (GATED) load8<ALIGNED>(v, z + a.cols, w.lane, n);
    if (a.a) {
      float o[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float s;
        act_and_slope<T, ACT>(g[k], o[k], s);
        if (GATED) o[k] *= v[k];
      }
      store8<ALIGNED>((T*)a.a + row * a.lda + w.at, o, w.lane, n);
    }
    float none;
    int8_t* q = a.q + row * a.ldq + w.at;
    float* sc = a.scales + row * a.lds + w.group;
    quantise<ALIGNED>(g, q, n > 0 ? sc : &none, w.lane, n);
    if (GATED) quantise<ALIGNED>(v, q + a.cols, n > 0 ? sc + a.groups : &none, w.lane, n);
  }
}

template <typename T, int ACT, bool GATED, bool ALIGNED>
__global__ void __launch_bounds__(THREADS) k_backward(const Args a) {
  pdl_enter();
  const Walk w = walk(a);
  if (w.n <= 0) return;
  for (int64_t row = w.row; row < a.rows; row += w.step) {
    const float* sc = a.scales + row * a.lds + w.group;
    const int8_t* q = a.q + row * a.ldq + w.at;
    float g[8], v[8], da[8], f[8], s[8];
    restore<ALIGNED>(g, q, sc[0], w.lane, w.n);
    if (GATED) restore<ALIGNED>(v, q + a.cols, sc[a.groups], w.lane, w.n);
    if (a.dz) load8<ALIGNED>(da, (const T*)a.da + row * a.ldda + w.at, w.lane, w.n);
#pragma unroll
    for (int k = 0; k < 8; ++k) act_and_slope<T, ACT>(g[k], f[k], s[k]);
    if (a.dz) {
      T* dz = (T*)a.dz + row * a.lddz + w.at;
      float o[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] = GATED ? da[k] * v[k] * s[k] : da[k] * s[k];
      store8<ALIGNED>(dz, o, w.lane, w.n);
      if (GATED) {
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = da[k] * f[k];
        store8<ALIGNED>(dz + a.cols, o, w.lane, w.n);
      }
    }
    if (a.a) {
      if (GATED)
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] *= v[k];
      store8<ALIGNED>((T*)a.a + row * a.lda + w.at, f, w.lane, w.n);
    }
  }
}

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(THREADS) k_restore(const Args a, int parts) {
  pdl_enter();
  const Walk w = walk(a);
  if (w.n <= 0) return;
  for (int64_t row = w.row; row < a.rows; row += w.step)
    for (int p = 0; p < parts; ++p) {
      float z[8];
      restore<ALIGNED>(z, a.q + row * a.ldq + (int64_t)p * a.cols + w.at, a.scales[row * a.lds + p * a.groups + w.group], w.lane, w.n);
      store8<ALIGNED>((T*)a.dz + row * a.lddz + (int64_t)p * a.cols + w.at, z, w.lane, w.n);
    }
}

// ------------------------------------------------------------------ host side
enum Pass { STORE, BACKWARD, RESTORE };

static dim3 grid_of(Args& a) {
  a.unit_cols = 1;
  while (a.unit_cols < UNITS && a.unit_cols < a.groups) a.unit_cols *= 2;
  const int deep = UNITS / a.unit_cols, gx = (a.groups + a.unit_cols - 1) / a.unit_cols;
  const int64_t rows = (a.rows + deep - 1) / deep;
  int64_t most = (int64_t)current_sm_count() * 32 / gx;       // four rounds of eight blocks per SM: long enough walks, no tail
  if (most < 1) most = 1;
  if (most > 65535) most = 65535;
  return dim3((unsigned)gx, (unsigned)(rows < most ? rows : most));
}
template <typename T, int ACT, bool GATED>
static void launch_act(Pass pass, dim3 grid, cudaStream_t s, const Args& a, bool aligned) {
  if (pass == STORE) {
    if (aligned) launch_pdl(k_store<T, ACT, GATED, true>, grid, dim3(THREADS), 0, s, a);
    else launch_pdl(k_store<T, ACT, GATED, false>, grid, dim3(THREADS), 0, s, a);
  } else {
    if (aligned) launch_pdl(k_backward<T, ACT, GATED, true>, grid, dim3(THREADS), 0, s, a);
    else launch_pdl(k_backward<T, ACT, GATED, false>, grid, dim3(THREADS), 0, s, a);
  }
}
template <typename T>
static betty_status launch(Pass pass, const betty_act8_cfg* c, Args& a, cudaStream_t s, bool aligned) {
  const dim3 grid = grid_of(a);
  if (pass == RESTORE) {
    if (aligned) launch_pdl(k_restore<T, true>, grid, dim3(THREADS), 0, s, a, c->gated ? 2 : 1);
    else launch_pdl(k_restore<T, false>, grid, dim3(THREADS), 0, s, a, c->gated ? 2 : 1);
  } else if (c->act == BETTY_ACT_RELU) {
    if (c->gated) launch_act<T, BETTY_ACT_RELU, true>(pass, grid, s, a, aligned); else launch_act<T, BETTY_ACT_RELU, false>(pass, grid, s, a, aligned);
  } else if (c->act == BETTY_ACT_GELU) {
    if (c->gated) launch_act<T, BETTY_ACT_GELU, true>(pass, grid, s, a, aligned); else launch_act<T, BETTY_ACT_GELU, false>(pass, grid, s, a, aligned);
  } else {
    if (c->gated) launch_act<T, BETTY_ACT_SILU, true>(pass, grid, s, a, aligned); else launch_act<T, BETTY_ACT_SILU, false>(pass, grid, s, a, aligned);
  }
  BETTY_LAUNCH_CHECK();
  return BETTY_OK;
}
static betty_status run(Pass pass, const betty_act8_cfg* c, Args& a, void* stream, bool aligned) {
  const cudaStream_t s = (cudaStream_t)stream;
  if (c->dtype == BETTY_F32) return launch<float>(pass, c, a, s, aligned);
  if (c->dtype == BETTY_BF16) return launch<__nv_bfloat16>(pass, c, a, s, aligned);
  return launch<__half>(pass, c, a, s, aligned);
}

static betty_status check_cfg(const betty_act8_cfg* c, int64_t rows) {
  if (!c || rows < 0 || c->act < BETTY_ACT_RELU || c->act > BETTY_ACT_SILU) return BETTY_ERR_INVALID_ARG;
  if (c->dtype != BETTY_F32 && c->dtype != BETTY_BF16 && c->dtype != BETTY_F16) return BETTY_ERR_DTYPE;
  if (c->cols < 1) return BETTY_ERR_SHAPE;
  if (c->cols > (1 << 29)) return BETTY_ERR_UNSUPPORTED;
  return BETTY_OK;
}
static betty_status check_matrix(const void* p, int64_t ld, int64_t rows, int64_t cols, int64_t bytes, int64_t access, bool& aligned) {
  if (!p) return BETTY_OK;
  if (rows > 1 && ld < cols) return BETTY_ERR_SHAPE;
  if ((uintptr_t)p % bytes) return BETTY_ERR_ALIGNMENT;
  if ((uintptr_t)p % access || (rows > 1 && (ld * bytes) % access)) aligned = false;
  return BETTY_OK;
}
static betty_status check_store(const betty_act8_cfg* c, int64_t rows, const int8_t* q, int64_t ldq, const float* scales, int64_t lds,
                                Args& a, bool& aligned) {
  const int parts = c->gated ? 2 : 1;
  if (!q || !scales) return BETTY_ERR_INVALID_ARG;
  a.rows = rows; a.cols = (int)c->cols; a.groups = (int)((c->cols + GROUP - 1) / GROUP);
  aligned = c->cols % 8 == 0;
  BETTY_TRY(check_matrix(q, ldq, rows, parts * c->cols, 1, 8, aligned));
  bool any = true;
  BETTY_TRY(check_matrix(scales, lds, rows, (int64_t)parts * a.groups, 4, 4, any));
  a.q = (int8_t*)q; a.ldq = ldq; a.scales = (float*)scales; a.lds = lds;
  return BETTY_OK;
}
static inline int64_t size_of(int dtype) { return dtype == BETTY_F32 ? 4 : 2; }

}  // namespace act8
}  // namespace betty

using namespace betty;
using namespace betty::act8;

extern "C" betty_status betty_act8_store(const betty_act8_cfg* cfg, int64_t rows, const void* z, int64_t ldz, void* act, int64_t lda,
                                         int8_t* q, int64_t ldq, float* scales, int64_t lds, void* stream) {
  BETTY_TRY(act8::check_cfg(cfg, rows));
  if (rows == 0) return BETTY_OK;
  if (!z) return BETTY_ERR_INVALID_ARG;
  Args a = {};
  bool aligned;
  const int64_t b = act8::size_of(cfg->dtype), width = cfg->cols * (cfg->gated ? 2 : 1);
  BETTY_TRY(check_store(cfg, rows, q, ldq, scales, lds, a, aligned));
  BETTY_TRY(act8::check_matrix(z, ldz, rows, width, b, 16, aligned));
  BETTY_TRY(act8::check_matrix(act, lda, rows, cfg->cols, b, 16, aligned));
  a.z = z; a.ldz = ldz; a.a = act; a.lda = lda;
  return run(STORE, cfg, a, stream, aligned);
}

extern "C" betty_status betty_act8_restore(const betty_act8_cfg* cfg, int64_t rows, const int8_t* q, int64_t ldq, const float* scales,
                                           int64_t lds, void* z, int64_t ldz, void* stream) {
  BETTY_TRY(act8::check_cfg(cfg, rows));
  if (rows == 0) return BETTY_OK;
  if (!z) return BETTY_ERR_INVALID_ARG;
  Args a = {};
  bool aligned;
  BETTY_TRY(check_store(cfg, rows, q, ldq, scales, lds, a, aligned));
  BETTY_TRY(act8::check_matrix(z, ldz, rows, cfg->cols * (cfg->gated ? 2 : 1), act8::size_of(cfg->dtype), 16, aligned));
  a.dz = z; a.lddz = ldz;
  return run(RESTORE, cfg, a, stream, aligned);
}

extern "C" betty_status betty_act8_backward(const betty_act8_cfg* cfg, int64_t rows, const int8_t* q, int64_t ldq, const float* scales,
                                            int64_t lds, const void* da, int64_t ldda, void* dz, int64_t lddz, void* act, int64_t lda,
                                            void* stream) {
  BETTY_TRY(act8::check_cfg(cfg, rows));
  if (rows == 0) return BETTY_OK;
  if ((!dz && !act) || (dz && !da)) return BETTY_ERR_INVALID_ARG;
  Args a = {};
  bool aligned;
  const int64_t b = act8::size_of(cfg->dtype);
  BETTY_TRY(check_store(cfg, rows, q, ldq, scales, lds, a, aligned));
  if (dz) BETTY_TRY(act8::check_matrix(da, ldda, rows, cfg->cols, b, 16, aligned));
  BETTY_TRY(act8::check_matrix(dz, lddz, rows, cfg->cols * (cfg->gated ? 2 : 1), b, 16, aligned));
  BETTY_TRY(act8::check_matrix(act, lda, rows, cfg->cols, b, 16, aligned));
  a.da = da; a.ldda = ldda; a.dz = dz; a.lddz = lddz; a.a = act; a.lda = lda;
  return run(BACKWARD, cfg, a, stream, aligned);
}
