// Forward pass of the block norm (see block_norm.cuh) and the C entry points.
#include "block_norm.cuh"

namespace betty {
namespace blocknorm {

// Bound by memory: per value of a 16-bit row 3 reads and 2 writes, ~20 operations.  Thread groups walk the rows with the
// parameters in registers and the next rows' values already on their way, R rows at a time: a row's own chain (values, sum,
// barrier, values, sum, barrier) is several times longer than the memory needs for it, and the rows of a batch share it.
template <typename TX, typename TY, int GR, bool PIPE, int CH, int R, bool GENERAL>
__global__ void __launch_bounds__(MAX_G, 1) k_forward(const Args a) {
  __shared__ float red[2 * RED_VALUES * 16];
  extern __shared__ __align__(16) char slots[];
  pdl_enter();
  const int G = a.G, d = a.d, t = threadIdx.x & (G - 1), sub = threadIdx.x / G, subs = blockDim.x / G;
  const int64_t step = (int64_t)gridDim.x * subs * R;
  int64_t row = ((int64_t)blockIdx.x * subs + sub) * R;
  const bool has_y = a.y != nullptr, has_g = a.gate != BETTY_GATE_NONE && has_y, has_u = a.u != nullptr;
  const int bytes_x = CH * 8 * G * (int)sizeof(TX), bytes_y = CH * 8 * G * (int)sizeof(TY);
  char* ring = slots + (size_t)sub * (a.ahead + 1) * R * a.slot_bytes;
  auto gate_row = [&](int64_t r) { return (const TY*)a.g + (a.per_gate == 1 ? r : (int64_t)((unsigned)r / a.per_gate)) * a.ldg; };
  auto fetch = [&](int64_t first, int slot) {
    if constexpr (PIPE) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int64_t r = first + i;
        if (r >= a.rows) break;
        char* p = ring + (slot * R + i) * a.slot_bytes;
        copy_row<GR, CH>(p, (const TX*)a.x + r * a.ldx, t, G, d);
        if (has_y) copy_row<GR, CH>(p + bytes_x, (const TY*)a.y + r * a.ldy, t, G, d);
        if (has_g) copy_row<GR, CH>(p + bytes_x + bytes_y, gate_row(r), t, G, d);
      }
      copies_commit();
    }
  };
  int half = 0, slot = 0;
  if (PIPE)
    for (int i = 0; i < a.ahead; ++i) fetch(row + i * step, i);
  float wp[CH][8], ws[CH][8], bp[GENERAL ? CH : 1][8], bs[GENERAL ? CH : 1][8];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    float s[8];
    load_param8<GR>(wp[c], a.params, c, t, G, d);
    load_param8<GR>(ws[c], a.params + d, c, t, G, d);
    load_param8<GR>(s, a.params + 2 * (int64_t)d, c, t, G, d);
    if (GENERAL) {
#pragma unroll
      for (int k = 0; k < 8; ++k) { bp[c][k] = 0.f; bs[c][k] = 0.f; }
      if (a.bias) {
        load_param8<GR>(bp[c], a.params + 3 * (int64_t)d, c, t, G, d);
        load_param8<GR>(bs[c], a.params + 4 * (int64_t)d, c, t, G, d);
      }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {      // the residual scale goes into the post-norm's parameters
      ws[c][k] *= s[k];
      if (GENERAL) bs[c][k] *= s[k];
    }
  }
  float mask[GENERAL ? CH : 1][8 / GR];      // 1 for columns of the row, 0 beyond it
  if (GENERAL)
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int k = 0; k < 8; k += GR) mask[c][k / GR] = column<GR>(c, k, t, G) < d ? 1.f : 0.f;
  // 1 / rms of each row (after its mean is taken off), or 1
  auto normalise = [&](float (&v)[R][CH][8], int kind, float (&r)[R]) {
    if (GENERAL && kind == BETTY_NORM_LAYER) {
      float s[R];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        s[i] = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int k = 0; k < 8; ++k) s[i] += v[i][c][k];
      }
      row_sums<R>(s, red, half, G, t);
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const float mean = s[i] * a.inv_d;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int k = 0; k < 8; ++k) v[i][c][k] = fmaf(-mean, mask[c][k / GR], v[i][c][k]);
      }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) r[i] = 1.f;
    if (kind != BETTY_NORM_NONE) {
      float s[R];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        s[i] = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int k = 0; k < 8; ++k) s[i] = fmaf(v[i][c][k], v[i][c][k], s[i]);
      }
      row_sums<R>(s, red, half, G, t);
#pragma unroll
      for (int i = 0; i < R; ++i) r[i] = rsqrtf(fmaf(s[i], a.inv_d, a.eps));
    }
  };
  for (; row < a.rows; row += step) {
    const char* p = nullptr;
    if (PIPE) {
      fetch(row + a.ahead * step, slot == 0 ? a.ahead : slot - 1);
      copies_wait(a.ahead);
      p = ring + slot * R * a.slot_bytes;
      slot = slot == a.ahead ? 0 : slot + 1;
    }
    float x[R][CH][8], y[R][CH][8], r[R];
    // rows past the last one hold whatever their slots hold; they take part in the sums and are not stored
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        if constexpr (PIPE) {
          read_slot<GR, TX>(x[i][c], p + i * a.slot_bytes, c, t, G);
          if (has_y) read_slot<GR, TY>(y[i][c], p + i * a.slot_bytes + bytes_x, c, t, G);
        } else {
          load8<GR>(x[i][c], (const TX*)a.x + row * a.ldx, c, t, G, d);
          if (has_y) load8<GR>(y[i][c], (const TY*)a.y + row * a.ldy, c, t, G, d);
        }
      }
    if (has_y) {
      normalise(y, a.post, r);
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          float g[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) g[k] = 1.f;
          if (has_g) {
            if constexpr (PIPE) read_slot<GR, TY>(g, p + i * a.slot_bytes + bytes_x + bytes_y, c, t, G);
            else load8<GR>(g, gate_row(row), c, t, G, d);
            if (a.gate == BETTY_GATE_SIGMOID)
#pragma unroll
              for (int k = 0; k < 8; ++k) g[k] = sigmoid_f(g[k]);
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float z = GENERAL ? fmaf(y[i][c][k] * r[i], ws[c][k], bs[c][k]) : y[i][c][k] * r[i] * ws[c][k];
            x[i][c][k] = fmaf(g[k], z, x[i][c][k]);
          }
          if (R == 1 || row + i < a.rows) store8<GR>((TX*)a.x_out + (row + i) * a.ldxo, x[i][c], c, t, G, d);
        }
    }
    if (has_u) {          // the entry norm reads x' before its rounding
      normalise(x, a.pre, r);
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          float o[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) o[k] = GENERAL ? fmaf(x[i][c][k] * r[i], wp[c][k], bp[c][k]) : x[i][c][k] * r[i] * wp[c][k];
          if (R == 1 || row + i < a.rows) store8<GR>((TY*)a.u + (row + i) * a.ldu, o, c, t, G, d);
        }
    }
  }
}

template <typename TX, typename TY, int GR, bool PIPE, int CH, int R, bool GENERAL>
static betty_status launch_forward(cudaStream_t stream, const Args& a, const Layout& l) {
  static SmemLimit limit = {};
  if (l.smem > 40 * 1024) BETTY_TRY(ensure_dynamic_smem(k_forward<TX, TY, GR, PIPE, CH, R, GENERAL>, limit, l.smem));
  const int per_block = l.threads / l.G * R;
  const int64_t want = (a.rows + per_block - 1) / per_block, most = (int64_t)l.blocks_per_sm * current_sm_count();
  launch_pdl(k_forward<TX, TY, GR, PIPE, CH, R, GENERAL>, dim3((unsigned)(want < most ? want : most)), dim3(l.threads), l.smem, stream, a);
  BETTY_LAUNCH_CHECK();
  return BETTY_OK;
}
// the wide kernel's chunks per thread and rows at a time: what 128 registers hold
static constexpr int FWD_CHUNKS = 2;
static constexpr int forward_batch(bool general) { return general ? 1 : 2; }
template <typename TX, typename TY, bool GENERAL>
static betty_status forward_layout(cudaStream_t stream, const Args& a, const Layout& l) {
  constexpr int R = forward_batch(GENERAL), CH = FWD_CHUNKS, GR = sizeof(TY) == 4 ? 1 : 2;
  if (l.granule == 8) {
    if (!l.ahead) return launch_forward<TX, TY, 8, false, 4, 1, GENERAL>(stream, a, l);
    return l.wide ? launch_forward<TX, TY, 8, true, CH, R, GENERAL>(stream, a, l) : launch_forward<TX, TY, 8, true, 1, 1, GENERAL>(stream, a, l);
  }
  if (!l.ahead) return launch_forward<TX, TY, 1, false, 4, 1, GENERAL>(stream, a, l);
  return l.wide ? launch_forward<TX, TY, GR, true, CH, R, GENERAL>(stream, a, l) : launch_forward<TX, TY, GR, true, 1, 1, GENERAL>(stream, a, l);
}
template <typename TX, typename TY>
static betty_status forward_typed(cudaStream_t stream, const Args& a, const Layout& l) {
  const bool general = a.bias || a.pre == BETTY_NORM_LAYER || a.post == BETTY_NORM_LAYER;
  return general ? forward_layout<TX, TY, true>(stream, a, l) : forward_layout<TX, TY, false>(stream, a, l);
}
betty_status forward(cudaStream_t stream, Args& a, int xd, int yd, int granule) {
  const int ys = (a.y ? 1 : 0) + (a.y && a.gate != BETTY_GATE_NONE ? 1 : 0);
  const bool general = a.bias || a.pre == BETTY_NORM_LAYER || a.post == BETTY_NORM_LAYER;
  const Layout l = layout_of(a.d, a.rows, xd, yd, granule, {1, ys, FWD_CHUNKS, forward_batch(general), 0, 0});
  a.G = l.G; a.ahead = l.ahead; a.slot_bytes = l.slot_bytes;
  if (xd == BETTY_F32 && yd == BETTY_F32) return forward_typed<float, float>(stream, a, l);
  if (xd == BETTY_F32 && yd == BETTY_BF16) return forward_typed<float, __nv_bfloat16>(stream, a, l);
  if (xd == BETTY_F32 && yd == BETTY_F16) return forward_typed<float, __half>(stream, a, l);
  if (xd == BETTY_BF16 && yd == BETTY_BF16) return forward_typed<__nv_bfloat16, __nv_bfloat16>(stream, a, l);
  return forward_typed<__half, __half>(stream, a, l);
}

// Many rows take the wide kernel (several chunks per thread: a row's fixed cost, its sums and addresses, is shared by more
// values); rows that would leave thread groups idle take one chunk per thread.  Rows that cannot be fetched ahead (16-bit
// values on odd addresses; rows so wide that two batches do not fit the shared memory) are read where they are used, four
// chunks per thread.
Layout layout_of(int64_t d, int64_t rows, int xd, int yd, int granule, const Needs& n) {
  const int bx = xd == BETTY_F32 ? 4 : 2, by = yd == BETTY_F32 ? 4 : 2, sms = current_sm_count();
  const bool pipe = granule == 8 || by == 4 || granule == 2;
  for (int attempt = pipe ? 0 : 2; ; ++attempt) {            // wide, one chunk per thread, not fetched ahead
    Layout l = {};
    l.granule = granule == 2 && by == 4 ? 1 : granule;
    l.wide = attempt == 0;
    l.chunks = attempt == 0 ? n.wide_chunks : (attempt == 1 ? 1 : MAX_CH);
    const int batch = attempt == 0 ? n.batch : 1;
    l.G = 32;
    while (l.G < MAX_G && (int64_t)l.G * 8 * l.chunks < d) l.G *= 2;
    if ((int64_t)l.G * 8 * l.chunks < d) continue;
    l.threads = l.G == 32 ? SMALL_THREADS : l.G;
    const int groups = l.threads / l.G;
    l.blocks_per_sm = MAX_G / l.threads;
    l.slot_bytes = l.chunks * 8 * l.G * (n.streams_x * bx + n.streams_y * by);
    const size_t acc = (size_t)(n.acc_arrays * groups + n.param_arrays) * l.chunks * 8 * l.G * sizeof(float);
    if (attempt == 2) {
      l.smem = acc;
      l.slot_bytes = 0;
      if (granule == 2) l.granule = 1;
      return l;
    }
    if (attempt == 0 && d <= (int64_t)MAX_G * 8 && rows < (int64_t)2 * batch * groups * l.blocks_per_sm * sms) continue;
    const int64_t slot = (int64_t)l.slot_bytes * groups * batch, budget = (int64_t)(222 * 1024) / l.blocks_per_sm - 2048 - (int64_t)acc;
    l.ahead = (int)(budget / slot) - 1;
    if (l.ahead < 1) continue;
    if (l.ahead > MAX_AHEAD) l.ahead = MAX_AHEAD;
    l.smem = acc + (size_t)(l.ahead + 1) * slot;
    return l;
  }
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
// a [rows, d] matrix: its stride covers a row and its address a value; `granule` (see block_norm.cuh) shrinks to what its
// rows' addresses allow
static betty_status check_matrix(const void* p, int64_t ld, int64_t rows, int64_t d, int dtype, int& granule) {
  if (!p) return BETTY_OK;
  if (rows > 1 && ld < d) return BETTY_ERR_SHAPE;
  const int64_t b = size_of(dtype), bytes = rows > 1 ? ld * b : 0;
  if ((uintptr_t)p % b) return BETTY_ERR_ALIGNMENT;
  if (granule == 8 && ((uintptr_t)p % 16 || bytes % 16)) granule = 2;
  if (granule == 2 && ((uintptr_t)p % 4 || bytes % 4)) granule = 1;
  return BETTY_OK;
}
static inline int widest_granule(int64_t d) { return d % 8 == 0 ? 8 : (d % 2 == 0 ? 2 : 1); }
static void common_args(Args& a, const betty_block_norm_cfg* c, int64_t rows, const float* params) {
  a.rows = rows; a.d = (int)c->d;
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
  int granule = widest_granule(d);
  BETTY_TRY(check_matrix(x, ldx, rows, d, cfg->x_dtype, granule));
  BETTY_TRY(check_matrix(y, ldy, rows, d, cfg->y_dtype, granule));
  if (y) BETTY_TRY(check_matrix(x_out, ldxo, rows, d, cfg->x_dtype, granule));
  if (y && cfg->gate != BETTY_GATE_NONE)
    BETTY_TRY(check_matrix(gate, ldg, (rows + cfg->rows_per_gate - 1) / cfg->rows_per_gate, d, cfg->y_dtype, granule));
  BETTY_TRY(check_matrix(u, ldu, rows, d, cfg->y_dtype, granule));
  Args a = {};
  common_args(a, cfg, rows, params);
  a.x = x; a.ldx = ldx; a.y = y; a.ldy = ldy; a.g = gate; a.ldg = ldg;
  a.x_out = x_out; a.ldxo = ldxo; a.u = u; a.ldu = ldu;
  return forward((cudaStream_t)stream, a, cfg->x_dtype, cfg->y_dtype, granule);
}

extern "C" betty_status betty_block_norm_workspace_size(const betty_block_norm_cfg* cfg, int64_t rows, size_t* bytes) {
  if (!bytes) return BETTY_ERR_INVALID_ARG;
  BETTY_TRY(check_cfg(cfg, rows));
  int64_t blocks = 0, walkers = 0;
  // whatever the matrices' types and addresses will be
  for (int granule : {8, 2, 1})
    for (int xd : {BETTY_F32, BETTY_BF16})
      for (int yd : {BETTY_F32, BETTY_BF16}) {
        const Layout l = backward_layout(cfg, rows, xd, yd, granule);
        const int64_t n = backward_blocks(rows, l), w = n * (l.threads / l.G);
        if (n > blocks) blocks = n;
        if (w > walkers) walkers = w;
      }
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
  int granule = widest_granule(d);
  if (rows > 0) {
    if ((!x_out && du) || (!du && !dx_out) || (!y && !du) || !dx || (y && !dy) || (gated && (!gate || !dgate))) return BETTY_ERR_INVALID_ARG;
    const int64_t gates = (rows + cfg->rows_per_gate - 1) / cfg->rows_per_gate;
    BETTY_TRY(check_matrix(x_out, ldxo, rows, d, cfg->x_dtype, granule));
    BETTY_TRY(check_matrix(y, ldy, rows, d, cfg->y_dtype, granule));
    BETTY_TRY(check_matrix(du, lddu, rows, d, cfg->y_dtype, granule));
    BETTY_TRY(check_matrix(dx_out, lddxo, rows, d, cfg->x_dtype, granule));
    BETTY_TRY(check_matrix(dx, lddx, rows, d, cfg->x_dtype, granule));
    if (y) BETTY_TRY(check_matrix(dy, lddy, rows, d, cfg->y_dtype, granule));
    if (gated) {
      BETTY_TRY(check_matrix(gate, ldg, gates, d, cfg->y_dtype, granule));
      BETTY_TRY(check_matrix(dgate, lddg, gates, d, cfg->y_dtype, granule));
    }
  }
  common_args(a, cfg, rows, params);
  if (!gated) a.gate = BETTY_GATE_NONE;
  a.x = x_out; a.ldx = ldxo; a.y = y; a.ldy = ldy; a.g = gate; a.ldg = ldg; a.du = du; a.lddu = lddu; a.dxo = dx_out; a.lddxo = lddxo;
  a.dx = dx; a.lddx = lddx; a.dy = dy; a.lddy = lddy; a.dg = dgate; a.lddg = lddg;
  Arena arena(ws, ws_bytes);
  const Layout l = backward_layout(cfg, rows, cfg->x_dtype, cfg->y_dtype, granule);
  const int blocks = backward_blocks(rows, l);
  a.walkers = blocks * (l.threads / l.G);         // as many as there are rows at most: no share is empty
  if (a.walkers > rows) a.walkers = rows > 0 ? (int)rows : 1;
  a.col_partials = arena.alloc<float>((size_t)blocks * quantities(cfg) * d);
  if (gated && cfg->rows_per_gate > 1)
    a.gate_partials = arena.alloc<float>((size_t)(a.walkers + (rows + cfg->rows_per_gate - 1) / cfg->rows_per_gate) * d);
  if (arena.overflow) return BETTY_ERR_WORKSPACE;
  return backward((cudaStream_t)stream, a, l, cfg->x_dtype, cfg->y_dtype, dparams);
}
