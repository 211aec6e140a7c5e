// Forward pass of the block norm (see block_norm.cuh) and the C entry points.
#include "block_norm.cuh"

namespace betty {
namespace blocknorm {

// Bound by memory: per value of a 16-bit row 3 reads and 2 writes, ~20 operations.  Thread groups walk the rows with the
// parameters in registers and the next row's values already requested while the present row is summed.
template <typename TX, typename TY, bool ALIGNED, int CH, bool GENERAL>
__global__ void __launch_bounds__(MAX_G) k_forward(const Args a) {
  __shared__ float red[2 * RED_VALUES * 32];
  pdl_enter();
  const int G = a.G, d = a.d, t = threadIdx.x & (G - 1);
  const int64_t step = (int64_t)gridDim.x * (blockDim.x / G);
  int64_t row = (int64_t)blockIdx.x * (blockDim.x / G) + threadIdx.x / G;
  const bool has_y = a.y != nullptr, has_g = a.gate != BETTY_GATE_NONE && has_y, has_u = a.u != nullptr;
  int half = 0;
  float wp[CH][8], ws[CH][8], bp[GENERAL ? CH : 1][8], bs[GENERAL ? CH : 1][8];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    float s[8];
    load_param8<ALIGNED>(wp[c], a.params, c, t, G, d);
    load_param8<ALIGNED>(ws[c], a.params + d, c, t, G, d);
    load_param8<ALIGNED>(s, a.params + 2 * (int64_t)d, c, t, G, d);
    if (GENERAL) {
#pragma unroll
      for (int k = 0; k < 8; ++k) { bp[c][k] = 0.f; bs[c][k] = 0.f; }
      if (a.bias) {
        load_param8<ALIGNED>(bp[c], a.params + 3 * (int64_t)d, c, t, G, d);
        load_param8<ALIGNED>(bs[c], a.params + 4 * (int64_t)d, c, t, G, d);
      }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {      // the residual scale goes into the post-norm's parameters
      ws[c][k] *= s[k];
      if (GENERAL) bs[c][k] *= s[k];
    }
  }
  Raw8<TX> xr[CH];
  Raw8<TY> yr[CH], gr[CH];
  auto request = [&](int64_t r) {
    const TX* x = (const TX*)a.x + r * a.ldx;
    const TY* y = (const TY*)a.y + r * a.ldy;
    const TY* g = has_g ? (const TY*)a.g + (int64_t)((unsigned)r / a.per_gate) * a.ldg : nullptr;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      load8<ALIGNED>(xr[c], x, c, t, G, d);
      if (has_y) load8<ALIGNED>(yr[c], y, c, t, G, d);
      if (has_g) load8<ALIGNED>(gr[c], g, c, t, G, d);
    }
  };
  if (row < a.rows) request(row);
  for (; row < a.rows; row += step) {
    float x[CH][8], y[CH][8], ag[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[c][k] = to_f(xr[c].v[k]);
        y[c][k] = has_y ? to_f(yr[c].v[k]) : 0.f;
        ag[c][k] = has_g ? to_f(gr[c].v[k]) : 1.f;
      }
    if (row + step < a.rows) request(row + step);
    if (has_y) {
      float mean = 0.f, r = 1.f;
      if (GENERAL && a.post == BETTY_NORM_LAYER) {
        float v[1] = {0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int k = 0; k < 8; ++k) v[0] += y[c][k];
        row_sums<1>(v, red, half, G, t);
        mean = v[0] * a.inv_d;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int k = 0; k < 8; ++k) y[c][k] = column<ALIGNED>(c, k, t, G) < d ? y[c][k] - mean : 0.f;
      }
      if (a.post != BETTY_NORM_NONE) {
        float v[1] = {0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int k = 0; k < 8; ++k) v[0] = fmaf(y[c][k], y[c][k], v[0]);
        row_sums<1>(v, red, half, G, t);
        r = rsqrtf(fmaf(v[0], a.inv_d, a.eps));
      }
      if (a.gate == BETTY_GATE_SIGMOID)
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int k = 0; k < 8; ++k) ag[c][k] = sigmoid_f(ag[c][k]);
      TX* xo = (TX*)a.x_out + row * a.ldxo;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float z = GENERAL ? fmaf(y[c][k] * r, ws[c][k], bs[c][k]) : y[c][k] * r * ws[c][k];
          x[c][k] = fmaf(ag[c][k], z, x[c][k]);
        }
        store8<ALIGNED>(xo, x[c], c, t, G, d);
      }
    }
    if (has_u) {          // the entry norm reads x' before its rounding
      float r = 1.f;
      if (GENERAL && a.pre == BETTY_NORM_LAYER) {
        float v[1] = {0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int k = 0; k < 8; ++k) v[0] += x[c][k];
        row_sums<1>(v, red, half, G, t);
        const float mean = v[0] * a.inv_d;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int k = 0; k < 8; ++k) x[c][k] = column<ALIGNED>(c, k, t, G) < d ? x[c][k] - mean : 0.f;
      }
      if (a.pre != BETTY_NORM_NONE) {
        float v[1] = {0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int k = 0; k < 8; ++k) v[0] = fmaf(x[c][k], x[c][k], v[0]);
        row_sums<1>(v, red, half, G, t);
        r = rsqrtf(fmaf(v[0], a.inv_d, a.eps));
      }
      TY* u = (TY*)a.u + row * a.ldu;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = GENERAL ? fmaf(x[c][k] * r, wp[c][k], bp[c][k]) : x[c][k] * r * wp[c][k];
        store8<ALIGNED>(u, o, c, t, G, d);
      }
    }
  }
}

template <typename TX, typename TY, bool ALIGNED, int CH, bool GENERAL>
static betty_status launch_forward(cudaStream_t stream, const Args& a) {
  const int threads = a.G == 32 ? SMALL_THREADS : a.G, per_block = threads / a.G;
  static std::atomic<int> resident[16];         // blocks per SM, by the logarithm of the block size
  int lg = 0;
  while ((1 << lg) < threads) ++lg;
  int occ = resident[lg].load(std::memory_order_relaxed);
  if (!occ) {
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&occ, k_forward<TX, TY, ALIGNED, CH, GENERAL>, threads, 0) != cudaSuccess || occ < 1) {
      (void)cudaGetLastError();
      return BETTY_ERR_CUDA;
    }
    resident[lg].store(occ, std::memory_order_relaxed);
  }
  const int64_t want = (a.rows + per_block - 1) / per_block, most = (int64_t)occ * current_sm_count();
  launch_pdl(k_forward<TX, TY, ALIGNED, CH, GENERAL>, dim3((unsigned)(want < most ? want : most)), dim3(threads), 0, stream, a);
  BETTY_LAUNCH_CHECK();
  return BETTY_OK;
}
template <typename TX, typename TY, bool ALIGNED, bool GENERAL>
static betty_status forward_chunks(cudaStream_t stream, const Args& a) {
  switch (chunks_of(a.d, a.G)) {
    case 1: return launch_forward<TX, TY, ALIGNED, 1, GENERAL>(stream, a);
    case 2: return launch_forward<TX, TY, ALIGNED, 2, GENERAL>(stream, a);
    default: return launch_forward<TX, TY, ALIGNED, 4, GENERAL>(stream, a);
  }
}
template <typename TX, typename TY>
static betty_status forward_typed(cudaStream_t stream, const Args& a, bool aligned) {
  const bool general = a.bias || a.pre == BETTY_NORM_LAYER || a.post == BETTY_NORM_LAYER;
  if (aligned) return general ? forward_chunks<TX, TY, true, true>(stream, a) : forward_chunks<TX, TY, true, false>(stream, a);
  return general ? forward_chunks<TX, TY, false, true>(stream, a) : forward_chunks<TX, TY, false, false>(stream, a);
}
betty_status forward(cudaStream_t stream, const Args& a, int xd, int yd, bool aligned) {
  if (xd == BETTY_F32 && yd == BETTY_F32) return forward_typed<float, float>(stream, a, aligned);
  if (xd == BETTY_F32 && yd == BETTY_BF16) return forward_typed<float, __nv_bfloat16>(stream, a, aligned);
  if (xd == BETTY_F32 && yd == BETTY_F16) return forward_typed<float, __half>(stream, a, aligned);
  if (xd == BETTY_BF16 && yd == BETTY_BF16) return forward_typed<__nv_bfloat16, __nv_bfloat16>(stream, a, aligned);
  return forward_typed<__half, __half>(stream, a, aligned);
}

// ------------------------------------------------------------------ arguments
static inline int64_t size_of(int dtype) { return dtype == BETTY_F32 ? 4 : 2; }

static betty_status check_cfg(const betty_block_norm_cfg* c, int64_t rows) {
  if (!c || rows < 0) return BETTY_ERR_INVALID_ARG;
  if (c->pre < BETTY_NORM_NONE || c->pre > BETTY_NORM_LAYER || c->post < BETTY_NORM_NONE || c->post > BETTY_NORM_LAYER ||
      c->gate < BETTY_GATE_NONE || c->gate > BETTY_GATE_SIGMOID || c->rows_per_gate < 1 || !(c->eps >= 0.f))
    return BETTY_ERR_INVALID_ARG;
  const int x = c->x_dtype, y = c->y_dtype;
  if (!((x == BETTY_F32 && (y == BETTY_F32 || y == BETTY_BF16 || y == BETTY_F16)) || (x == y && (x == BETTY_BF16 || x == BETTY_F16))))
    return BETTY_ERR_DTYPE;
  if (c->d < 1) return BETTY_ERR_SHAPE;
  if (c->d > MAX_D || rows > INT32_MAX || c->rows_per_gate > INT32_MAX) return BETTY_ERR_UNSUPPORTED;
  return BETTY_OK;
}
// a [rows, d] matrix: its stride covers a row and its address a value; `aligned` is cleared when 16-byte accesses do not fit
static betty_status check_matrix(const void* p, int64_t ld, int64_t rows, int64_t d, int dtype, bool& aligned) {
  if (!p) return BETTY_OK;
  if (rows > 1 && ld < d) return BETTY_ERR_SHAPE;
  const int64_t b = size_of(dtype);
  if ((uintptr_t)p % b) return BETTY_ERR_ALIGNMENT;
  if (!aligned16(p) || (rows > 1 && (ld * b) % 16)) aligned = false;
  return BETTY_OK;
}
static void common_args(Args& a, const betty_block_norm_cfg* c, int64_t rows, const float* params) {
  a.rows = rows; a.d = (int)c->d; a.G = threads_per_row(c->d);
  a.pre = c->pre; a.post = c->post; a.gate = c->gate; a.bias = c->bias != 0;
  a.per_gate = (unsigned)c->rows_per_gate;
  a.eps = c->eps; a.inv_d = 1.f / (float)c->d; a.params = params;
}
static inline int quantities(const betty_block_norm_cfg* c) { return c->bias ? 4 : 2; }

}  // namespace blocknorm
}  // namespace betty

using namespace betty;
using namespace betty::blocknorm;

extern "C" betty_status betty_block_norm(const betty_block_norm_cfg* cfg, const float* params, int64_t rows, const void* x,
                                         int64_t ldx, const void* y, int64_t ldy, const void* gate, int64_t ldg, void* x_out,
                                         int64_t ldxo, void* u, int64_t ldu, void* stream) {
  BETTY_TRY(check_cfg(cfg, rows));
  if (rows == 0) return BETTY_OK;
  if (!params || !x || (!y && !u) || (y && !x_out) || (y && cfg->gate != BETTY_GATE_NONE && !gate)) return BETTY_ERR_INVALID_ARG;
  if (!aligned16(params)) return BETTY_ERR_ALIGNMENT;
  const int64_t d = cfg->d;
  bool aligned = d % 8 == 0;
  BETTY_TRY(check_matrix(x, ldx, rows, d, cfg->x_dtype, aligned));
  BETTY_TRY(check_matrix(y, ldy, rows, d, cfg->y_dtype, aligned));
  if (y) BETTY_TRY(check_matrix(x_out, ldxo, rows, d, cfg->x_dtype, aligned));
  if (y && cfg->gate != BETTY_GATE_NONE)
    BETTY_TRY(check_matrix(gate, ldg, (rows + cfg->rows_per_gate - 1) / cfg->rows_per_gate, d, cfg->y_dtype, aligned));
  BETTY_TRY(check_matrix(u, ldu, rows, d, cfg->y_dtype, aligned));
  Args a = {};
  common_args(a, cfg, rows, params);
  a.x = x; a.ldx = ldx; a.y = y; a.ldy = ldy; a.g = gate; a.ldg = ldg;
  a.x_out = x_out; a.ldxo = ldxo; a.u = u; a.ldu = ldu;
  return forward((cudaStream_t)stream, a, cfg->x_dtype, cfg->y_dtype, aligned);
}

extern "C" betty_status betty_block_norm_workspace_size(const betty_block_norm_cfg* cfg, int64_t rows, size_t* bytes) {
  if (!bytes) return BETTY_ERR_INVALID_ARG;
  BETTY_TRY(check_cfg(cfg, rows));
  const int G = threads_per_row(cfg->d);
  const int64_t blocks = backward_blocks(rows, G), walkers = blocks * (G == 32 ? SMALL_THREADS / 32 : 1);
  const int64_t gates = (rows + cfg->rows_per_gate - 1) / cfg->rows_per_gate;
  int64_t floats = blocks * quantities(cfg) * cfg->d;
  if (cfg->gate != BETTY_GATE_NONE && cfg->rows_per_gate > 1) floats += (walkers + gates) * cfg->d;
  *bytes = sizeof(StatusBlock) + 2 * 256 + (size_t)floats * sizeof(float);
  return BETTY_OK;
}

extern "C" betty_status betty_block_norm_backward(const betty_block_norm_cfg* cfg, const float* params, int64_t rows,
                                                  const void* x_out, int64_t ldxo, const void* y, int64_t ldy, const void* gate,
                                                  int64_t ldg, const void* du, int64_t lddu, const void* dx_out, int64_t lddxo,
                                                  void* dx, int64_t lddx, void* dy, int64_t lddy, void* dgate, int64_t lddg,
                                                  float* dparams, void* ws, size_t ws_bytes, void* stream) {
  BETTY_TRY(check_cfg(cfg, rows));
  if (!params || !dparams) return BETTY_ERR_INVALID_ARG;
  if (!aligned16(params) || !aligned16(dparams)) return BETTY_ERR_ALIGNMENT;
  if (!ws || ws_bytes < sizeof(StatusBlock) || (((uintptr_t)ws) & 255u)) return BETTY_ERR_WORKSPACE;
  const int64_t d = cfg->d;
  const bool gated = y && cfg->gate != BETTY_GATE_NONE;
  Args a = {};
  bool aligned = d % 8 == 0;
  if (rows > 0) {
    if ((!x_out && du) || (!du && !dx_out) || (!y && !du) || !dx || (y && !dy) || (gated && (!gate || !dgate))) return BETTY_ERR_INVALID_ARG;
    const int64_t gates = (rows + cfg->rows_per_gate - 1) / cfg->rows_per_gate;
    BETTY_TRY(check_matrix(x_out, ldxo, rows, d, cfg->x_dtype, aligned));
    BETTY_TRY(check_matrix(y, ldy, rows, d, cfg->y_dtype, aligned));
    BETTY_TRY(check_matrix(du, lddu, rows, d, cfg->y_dtype, aligned));
    BETTY_TRY(check_matrix(dx_out, lddxo, rows, d, cfg->x_dtype, aligned));
    BETTY_TRY(check_matrix(dx, lddx, rows, d, cfg->x_dtype, aligned));
    if (y) BETTY_TRY(check_matrix(dy, lddy, rows, d, cfg->y_dtype, aligned));
    if (gated) {
      BETTY_TRY(check_matrix(gate, ldg, gates, d, cfg->y_dtype, aligned));
      BETTY_TRY(check_matrix(dgate, lddg, gates, d, cfg->y_dtype, aligned));
    }
  }
  common_args(a, cfg, rows, params);
  if (!gated) a.gate = BETTY_GATE_NONE;
  a.x = x_out; a.ldx = ldxo; a.y = y; a.ldy = ldy; a.g = gate; a.ldg = ldg; a.du = du; a.lddu = lddu; a.dxo = dx_out; a.lddxo = lddxo;
  a.dx = dx; a.lddx = lddx; a.dy = dy; a.lddy = lddy; a.dg = dgate; a.lddg = lddg;
  Arena arena(ws, ws_bytes);
  const int blocks = backward_blocks(rows, a.G);
  a.walkers = blocks * (a.G == 32 ? SMALL_THREADS / 32 : 1);
  a.col_partials = arena.alloc<float>((size_t)blocks * quantities(cfg) * d);
  if (gated && cfg->rows_per_gate > 1)
    a.gate_partials = arena.alloc<float>((size_t)(a.walkers + (rows + cfg->rows_per_gate - 1) / cfg->rows_per_gate) * d);
  if (arena.overflow) return BETTY_ERR_WORKSPACE;
  return backward((cudaStream_t)stream, a, cfg->x_dtype, cfg->y_dtype, aligned, dparams);
}
