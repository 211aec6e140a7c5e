// 8-bit checkpoints of a hidden layer's pre-activations, and the layer's backward pass from them.
//
// A row of z (or each half of a gated row [gate | value]) is cut into groups of 128 values.  A group is held as whole
// numbers in [-127, 127] and one fp32 scale:
//
//   top = max |z|,   q = rint(z * (127 * (1 / top))),   scale = top * (1 / 127),   z~ = q * scale
//
// every operation rounded to fp32 on its own (no contraction, a subnormal 1 / top kept), so that q is the same whoever computes it.
// A group whose top is below 1e-30 is held as zeros; one that holds an infinity or a NaN gets the scale NaN, so that it stays visible.
//
//   store:     a = act(z)                 or  act(z_gate) * z_value;  z -> q, scale
//   backward:  dz = da * act'(z~)         or  [da * z~_value * act'(z~_gate) | da * act(z~_gate)];   a from z~ for the
//              weight gradient of the next layer, which so needs no stored activation either
//
// Backward and restore are bound by memory; the store also by its instructions (5 bytes per value at ~25 operations), so
// rounding and the bytes' conversion go through additions of 1.5 * 2^23 and byte permutes, not through the conversion
// instructions, which share the special-function pipe with exp and the reciprocal, and values are worked on in pairs.
// Measured: 16384 x 4096 bf16, GELU: store 72 us (bytes alone 52), restore 43 (31); 8192 x 8192 fp16, gated SiLU, backward 117 us
// (104, 5.8 TB/s).
#include "gemm.cuh"
#include "values.cuh"

namespace betty {
namespace act8 {

static constexpr int GROUP = 128;
static constexpr int LANES = 16;              // backward, restore: half a warp holds a group, 8 values per lane
static constexpr int STORE_LANES = 8;         // store: a quarter, 16 values per lane (what a group costs besides is shared by more)
static constexpr int THREADS = 256;
static constexpr float TINY = 1e-30f;

struct Args {
  int64_t rows;
  int cols, groups;        // per part
  int unit_cols;           // groups of one row a block holds side by side (a power of two)
  const void* z; uint32_t ldz;
  void* a; uint32_t lda;
  int8_t* q; uint32_t ldq;
  float* scales; uint32_t lds;
  const void* da; uint32_t ldda;
  void* dz; uint32_t lddz;
};

template <typename T> struct alignas(16) Raw8 { T v[8]; };

// Lane l of a group's lanes holds its values 8l .. 8l+7 where rows allow 16-byte accesses, else l, l + LANES, ...

// zeros for the places from n on
template <bool ALIGNED, int LANES, typename T>
__device__ __forceinline__ void load_raw(Raw8<T>& r, const T* row, int lane, int n) {
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
}
template <bool ALIGNED, typename T>
__device__ __forceinline__ void values_of(f2 (&v)[4], const Raw8<T>& r) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (sizeof(T) == 4) v[k] = f2{r.v[2 * k], r.v[2 * k + 1]};
    else unpack2<T>(((const uint32_t*)r.v)[k], v[k].x, v[k].y);
  }
}
template <bool ALIGNED, int LANES, typename T>
__device__ __forceinline__ void store8(T* row, const f2 (&v)[4], int lane, int n) {
  if (ALIGNED) {
    if (lane * 8 < n) {
      if constexpr (sizeof(T) == 4) {
        *(float4*)(row + lane * 8) = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
        *(float4*)(row + lane * 8 + 4) = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
      } else {
        *(uint4*)(row + lane * 8) = make_uint4(pack2<T>(v[0].x, v[0].y), pack2<T>(v[1].x, v[1].y), pack2<T>(v[2].x, v[2].y), pack2<T>(v[3].x, v[3].y));
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (lane + k * LANES < n) row[lane + k * LANES] = from_f<T>(k & 1 ? v[k / 2].y : v[k / 2].x);
  }
}

__device__ __forceinline__ float max_nan(float a, float b) {       // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// 127 * (1 / t), both operations rounded to fp32 with subnormal results kept: 1 / t is one from t = 2^126 on (the library is
// compiled with subnormals flushed, which would make the whole group zeros), the product never is
__device__ __forceinline__ float steps_per_unit(float t) {
  float r;
  asm("{\n\t.reg .f32 a;\n\trcp.rn.f32 a, %1;\n\tmul.rn.f32 %0, a, 0f42FE0000;\n\t}" : "=f"(r) : "f"(t));
  return r;
}
// z -> q (its fp32 holder's low byte) and the group's scale; lane l of a group's STORE_LANES lanes has its values 8l .. 8l+7 and
// 64 + 8l .. (aligned rows; otherwise every STORE_LANES-th of each half)
template <bool ALIGNED>
__device__ __forceinline__ void quantise(const f2 (&z)[2][4], int8_t* q, float* scale, int lane, int n) {
  float t = 0.f;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int k = 0; k < 4; ++k) t = max_nan(max_nan(t, fabsf(z[h][k].x)), fabsf(z[h][k].y));
#pragma unroll
  for (int o = STORE_LANES / 2; o; o >>= 1) t = max_nan(t, __shfl_xor_sync(0xffffffffu, t, o));
  const bool bad = !(t <= 3.4028235e38f), some = t >= TINY && !bad;
  const float inv = some ? steps_per_unit(t) : 0.f;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t b[8];
    // a product and a sum, each rounded (pairs would be contracted): adding 1.5 * 2^23 leaves the nearest whole number in
    // the low bits
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      b[2 * k] = __float_as_uint(__fadd_rn(__fmul_rn(z[h][k].x, inv), 12582912.f));
      b[2 * k + 1] = __float_as_uint(__fadd_rn(__fmul_rn(z[h][k].y, inv), 12582912.f));
    }
    if (!some)
#pragma unroll
      for (int k = 0; k < 8; ++k) b[k] = 0u;
    int8_t* to = q + h * 64;
    const int left = n - h * 64;
    if (ALIGNED) {
      if (lane * 8 < left) {
        uint2 w;
        w.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
        w.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
        *(uint2*)(to + lane * 8) = w;
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (lane + k * STORE_LANES < left) to[lane + k * STORE_LANES] = (int8_t)(b[k] & 0xffu);
    }
  }
  if (lane == 0 && n > 0) *scale = bad ? __uint_as_float(0x7fffffffu) : (some ? __fmul_rn(t, 1.f / 127.f) : 0.f);
}
// eight values of a checkpoint as they are held, and as fp32
template <bool ALIGNED> struct Held {
  uint32_t w[2];
  float scale;
  __device__ __forceinline__ void load(const int8_t* q, const float* sc, int lane, int n) {
    w[0] = w[1] = 0;
    scale = 0.f;
    if (n <= 0) return;
    scale = *sc;
    if (ALIGNED) {
      if (lane * 8 < n) { const uint2 v = *(const uint2*)(q + lane * 8); w[0] = v.x; w[1] = v.y; }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (lane + k * LANES < n) w[k >> 2] |= (uint32_t)(uint8_t)q[lane + k * LANES] << (8 * (k & 3));
    }
  }
  __device__ __forceinline__ void values(f2 (&z)[4]) const {
    const uint32_t u[2] = {w[0] ^ 0x80808080u, w[1] ^ 0x80808080u};     // q + 128, a byte that becomes the low bits of 2^23 + q + 128
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t x = u[k >> 1];
      const f2 f = {__uint_as_float(__byte_perm(x, 0x4b000000u, 0x7650 + (2 * k & 3))), __uint_as_float(__byte_perm(x, 0x4b000000u, 0x7651 + (2 * k & 3)))};
      z[k] = mul2(add2(f, both(-8388736.f)), both(scale));
    }
  }
};

// Activation and its slope (each used where the caller uses it).  fp32 values take erff, whose 1 + erf has 6e-8 absolute error.
// For 16-bit types the distribution function of -|v| is exp(-v^2 / 2) t (c0 + c1 t + .. + c5 t^5), t = 1 / (1 + 0.31 |v|): its ratio
// to the density is smooth and of order t, and the six coefficients are the ones of smallest largest RELATIVE error on 0 <= |v| <= 16
// (4.6e-6, a linear program over 3000 points).  So the activation of negative values keeps its bits as far down as the type
// holds it: 8e-6 of itself to v = -9, 2e-5 to -13, against 2^-12 and 2^-9 of the rounding; with a bound on the absolute error alone it
// was off by 4 to 54 units of the last place between -4 and -6.  The exponential is the slope's, too.
template <typename T, int ACT>
__device__ __forceinline__ void act_and_slope(f2 v, f2& f, f2& s) {
  if (ACT == BETTY_ACT_RELU) {
    f = f2{v.x != v.x ? v.x : fmaxf(v.x, 0.f), v.y != v.y ? v.y : fmaxf(v.y, 0.f)};
    s = f2{v.x != v.x ? v.x : (v.x > 0.f ? 1.f : 0.f), v.y != v.y ? v.y : (v.y > 0.f ? 1.f : 0.f)};
  } else if (ACT == BETTY_ACT_SILU) {
    f2 e, rest;              // the sigmoid and 1 - it
    if constexpr (sizeof(T) == 4) {
      sigmoid_parts(v.x, e.x, rest.x);
      sigmoid_parts(v.y, e.y, rest.y);
    } else {                 // within 2^-22 (2 + |v|) of itself, against 2^-12 and 2^-9 of the rounding
      e = f2{__fdividef(1.f, 1.f + __expf(-v.x)), __fdividef(1.f, 1.f + __expf(-v.y))};
      rest = fma2(e, both(-1.f), both(1.f));
    }
    f = mul2(v, e);
    s = mul2(e, fma2(v, rest, both(1.f)));
  } else {
    f2 c, density;
    if constexpr (sizeof(T) == 4) {
      c = f2{0.5f * (1.f + erff(v.x * 0.7071067811865476f)), 0.5f * (1.f + erff(v.y * 0.7071067811865476f))};
      density = f2{fam_bf16::norm_pdf(v.x), fam_bf16::norm_pdf(v.y)};
    } else {
      const f2 w = fma2(f2{fabsf(v.x), fabsf(v.y)}, both(0.31f), both(1.f)), t = {reciprocal(w.x), reciprocal(w.y)};
      const f2 power = mul2(mul2(v, v), both(-0.7213475204444817f)), e = {exp2_f(power.x), exp2_f(power.y)};     // -v^2 / 2 / ln 2
      f2 p = fma2(t, both(-0.0739143044f), both(0.180404842f));
      p = fma2(p, t, both(0.0157973096f));
      p = fma2(p, t, both(0.133401588f));
      p = fma2(p, t, both(0.12044815f));
      p = fma2(p, t, both(0.123860106f));
      const f2 h = mul2(mul2(p, t), e);            // the smaller tail
      c = f2{v.x >= 0.f ? 1.f - h.x : h.x, v.y >= 0.f ? 1.f - h.y : h.y};
      density = mul2(e, both(0.3989422804014327f));
    }
    f = mul2(v, c);
    s = fma2(v, density, c);
  }
}

// A block holds unit_cols groups of `deep` rows side by side; a thread keeps its columns and takes BATCH rows at a time, all of
// whose loads are issued before the first is used: what is in flight per SM, not arithmetic, is what bounds these kernels.
// Units without a group and rows past the last one load nothing and store nothing but stay in the shuffles.
struct Walk { int lane, group, at, n; int64_t row, step; };
template <int LANES>
__device__ __forceinline__ Walk walk(const Args& a) {
  Walk w;
  const int unit = threadIdx.x / LANES, deep = THREADS / LANES / a.unit_cols;
  w.lane = threadIdx.x & (LANES - 1);
  w.group = blockIdx.x * a.unit_cols + (unit & (a.unit_cols - 1));
  w.at = w.group * GROUP;
  w.n = min(GROUP, a.cols - w.at);                   // <= 0: no group
  w.row = (int64_t)blockIdx.y * deep + unit / a.unit_cols;
  w.step = (int64_t)gridDim.y * deep;
  return w;
}
template <typename T, bool GATED, bool ALIGNED> struct Batch { static constexpr int rows = !ALIGNED ? 1 : (sizeof(T) == 2 ? 4 : 2) / (GATED ? 2 : 1); };

template <typename T, int ACT, bool GATED, bool ALIGNED>
__global__ void __launch_bounds__(THREADS) k_store(const Args a) {
  constexpr int R = Batch<T, GATED, ALIGNED>::rows > 1 ? Batch<T, GATED, ALIGNED>::rows / 2 : 1;
  pdl_enter();
  const Walk w = walk<STORE_LANES>(a);
  const int deep = THREADS / STORE_LANES / a.unit_cols;
  // the block's first row decides, so that whole warps stay together
  for (int64_t base = (int64_t)blockIdx.y * deep; base < a.rows; base += R * w.step) {
    const int64_t row0 = w.row + (base - (int64_t)blockIdx.y * deep);
    Raw8<T> gr[R][2], vr[GATED ? R : 1][2];
    int n[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int64_t row = row0 + i * w.step;
      n[i] = row < a.rows && w.n > 0 ? w.n : 0;
      const T* z = row_at<T>(a.z, n[i] ? row : 0, a.ldz) + w.at;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        load_raw<ALIGNED, STORE_LANES>(gr[i][h], z + h * 64, w.lane, n[i] - h * 64);
        if (GATED) load_raw<ALIGNED, STORE_LANES>(vr[GATED ? i : 0][h], z + a.cols + h * 64, w.lane, n[i] - h * 64);
      }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int64_t row = n[i] ? row0 + i * w.step : 0;
      f2 g[2][4], v[2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        values_of<ALIGNED>(g[h], gr[i][h]);
        if (GATED) values_of<ALIGNED>(v[h], vr[GATED ? i : 0][h]);
        if (a.a) {
          f2 o[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            f2 s;
            act_and_slope<T, ACT>(g[h][k], o[k], s);
            if (GATED) o[k] = mul2(o[k], v[h][k]);
          }
          store8<ALIGNED, STORE_LANES>(row_at<T>(a.a, row, a.lda) + w.at + h * 64, o, w.lane, n[i] - h * 64);
        }
      }
      int8_t* q = row_at<int8_t>((void*)a.q, row, a.ldq) + w.at;
      float* sc = row_at<float>((void*)a.scales, row, a.lds) + w.group;
      quantise<ALIGNED>(g, q, sc, w.lane, n[i]);
      if (GATED) quantise<ALIGNED>(v, q + a.cols, sc + a.groups, w.lane, n[i]);
    }
  }
}

template <typename T, int ACT, bool GATED, bool ALIGNED>
__global__ void __launch_bounds__(THREADS) k_backward(const Args a) {
  constexpr int R = Batch<T, GATED, ALIGNED>::rows;
  pdl_enter();
  const Walk w = walk<LANES>(a);
  if (w.n <= 0) return;
  for (int64_t row0 = w.row; row0 < a.rows; row0 += R * w.step) {
    Held<ALIGNED> g[R], v[GATED ? R : 1];
    Raw8<T> da[R];
    int n[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int64_t row = row0 + i * w.step;
      n[i] = row < a.rows ? w.n : 0;
      const int64_t at = n[i] ? row : 0;
      const int8_t* q = row_at<int8_t>((const void*)a.q, at, a.ldq) + w.at;
      const float* sc = row_at<float>((const void*)a.scales, at, a.lds) + w.group;
      g[i].load(q, sc, w.lane, n[i]);
      if (GATED) v[GATED ? i : 0].load(q + a.cols, sc + a.groups, w.lane, n[i]);
      if (a.dz) load_raw<ALIGNED, LANES>(da[i], row_at<T>(a.da, at, a.ldda) + w.at, w.lane, n[i]);
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int64_t row = row0 + i * w.step;
      f2 z[4], u[4], f[4], s[4], d[4], o[4];
      g[i].values(z);
      if (GATED) v[GATED ? i : 0].values(u);
#pragma unroll
      for (int k = 0; k < 4; ++k) act_and_slope<T, ACT>(z[k], f[k], s[k]);
      if (a.dz) {
        T* dz = row_at<T>(a.dz, row, a.lddz) + w.at;
        values_of<ALIGNED>(d, da[i]);
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = GATED ? mul2(mul2(d[k], u[k]), s[k]) : mul2(d[k], s[k]);
        store8<ALIGNED, LANES>(dz, o, w.lane, n[i]);
        if (GATED) {
#pragma unroll
          for (int k = 0; k < 4; ++k) o[k] = mul2(d[k], f[k]);
          store8<ALIGNED, LANES>(dz + a.cols, o, w.lane, n[i]);
        }
      }
      if (a.a) {
        if (GATED)
#pragma unroll
          for (int k = 0; k < 4; ++k) f[k] = mul2(f[k], u[k]);
        store8<ALIGNED, LANES>(row_at<T>(a.a, row, a.lda) + w.at, f, w.lane, n[i]);
      }
    }
  }
}

// part p of a row: blockIdx.z
template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(THREADS) k_restore(const Args a) {
  constexpr int R = ALIGNED ? 2 : 1;
  pdl_enter();
  const Walk w = walk<LANES>(a);
  const int p = blockIdx.z;
  if (w.n <= 0) return;
  for (int64_t row0 = w.row; row0 < a.rows; row0 += R * w.step) {
    Held<ALIGNED> g[R];
    int n[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int64_t row = row0 + i * w.step;
      n[i] = row < a.rows ? w.n : 0;
      const int64_t at = n[i] ? row : 0;
      g[i].load(row_at<int8_t>((const void*)a.q, at, a.ldq) + (int64_t)p * a.cols + w.at, row_at<float>((const void*)a.scales, at, a.lds) + p * a.groups + w.group,
                w.lane, n[i]);
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      f2 z[4];
      g[i].values(z);
      store8<ALIGNED, LANES>(row_at<T>(a.dz, row0 + i * w.step, a.lddz) + (int64_t)p * a.cols + w.at, z, w.lane, n[i]);
    }
  }
}

// ------------------------------------------------------------------ host side
enum Pass { STORE, BACKWARD, RESTORE };

static dim3 grid_of(Pass pass, Args& a) {
  const int units = THREADS / (pass == STORE ? STORE_LANES : LANES);
  a.unit_cols = 1;
  while (a.unit_cols < units && a.unit_cols < a.groups) a.unit_cols *= 2;
  const int deep = units / a.unit_cols, gx = (a.groups + a.unit_cols - 1) / a.unit_cols;
  const int64_t rows = (a.rows + deep - 1) / deep;
  // walks of a few batches each.  Measured at 16384 x 4096 bf16: restore 55.6 us with 16 blocks per SM and 8 rows at a time, 43.0
  // with 64 and 2; store and backward (8192 x 2 x 8192 fp16) 3 to 15 % faster with 16 and 4 than with 64 or 128 and 2
  int64_t most = (int64_t)current_sm_count() * (pass == RESTORE ? 64 : 16) / gx;
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
  const dim3 grid = grid_of(pass, a);
  if (pass == RESTORE) {
    const dim3 parts(grid.x, grid.y, c->gated ? 2 : 1);
    if (aligned) launch_pdl(k_restore<T, true>, parts, dim3(THREADS), 0, s, a);
    else launch_pdl(k_restore<T, false>, parts, dim3(THREADS), 0, s, a);
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
  if (c->cols > (1 << 28) || rows > INT32_MAX) return BETTY_ERR_UNSUPPORTED;
  return BETTY_OK;
}
static betty_status check_matrix(const void* p, int64_t ld, int64_t rows, int64_t cols, int64_t bytes, int64_t access, bool& aligned) {
  if (!p) return BETTY_OK;
  if (rows > 1 && ld < cols) return BETTY_ERR_SHAPE;
  if (rows > 1 && ld >= (1 << 30)) return BETTY_ERR_UNSUPPORTED;      // row addresses take 32-bit numbers and strides in bytes
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
  a.q = (int8_t*)q; a.ldq = (uint32_t)ldq; a.scales = (float*)scales; a.lds = (uint32_t)lds * 4;
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
  a.z = z; a.ldz = (uint32_t)(ldz * b); a.a = act; a.lda = (uint32_t)(lda * b);
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
  a.dz = z; a.lddz = (uint32_t)(ldz * act8::size_of(cfg->dtype));
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
  a.da = da; a.ldda = (uint32_t)(ldda * b); a.dz = dz; a.lddz = (uint32_t)(lddz * b); a.a = act; a.lda = (uint32_t)(lda * b);
  return run(BACKWARD, cfg, a, stream, aligned);
}
