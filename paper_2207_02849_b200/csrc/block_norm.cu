// Forward pass of the block norm (see block_norm.cuh) and the C entry points.
#include "block_norm.cuh"

namespace betty {
namespace blocknorm {

// Bound by memory: per value of a 16-bit row 3 reads and 2 writes, ~20 operations.  Thread groups walk the rows with the
// parameters in registers and the next rows' values already on their way, R rows at a time: a row's own chain (values, sum,
// barrier, values, sum, barrier) is several times longer than the memory needs for it, and the rows of a batch share it.
// Measured at 16384 x 4096 bf16 with a gate per row: 180 us with one row per 512 threads and the next one in registers, 140 with
// four rows at a time, 108 to 120 with two rows of two chunks in each of two blocks per SM (5.6 to 6.2 TB/s; the bytes
// alone 104 us).
template <typename TX, typename TY, bool VEC, int CH, int R, bool GENERAL>
__global__ void __launch_bounds__(MAX_G, 1) k_forward(const Args a) {
  __shared__ __align__(16) float red[2 * RED_VALUES * 16];
  extern __shared__ __align__(16) char slots[];
  row_sums_init(red);
  pdl_enter();
  const int G = a.G, d = a.d, t = G == 32 ? threadIdx.x & 31 : threadIdx.x, sub = G == 32 ? threadIdx.x >> 5 : 0, subs = G == 32 ? blockDim.x >> 5 : 1;
  // thread group `g` takes rows kind, kind + classes, ... : batches g / classes, g / classes + step, ... of R of them
  const int g_id = blockIdx.x * subs + sub, kind = g_id % a.classes;
  const int64_t n_rows = (a.rows - kind + a.classes - 1) / a.classes, step = (int64_t)(gridDim.x * subs / a.classes) * R;
  int64_t at = g_id < (int)(gridDim.x * subs / a.classes) * a.classes ? (int64_t)(g_id / a.classes) * R : n_rows;
  const Place w = {t, G, d, VEC ? (int)((kind * a.ld8) & 7) : 0};
  auto row_of = [&](int64_t i) { return kind + i * a.classes; };
  const bool has_y = a.y != nullptr, has_g = a.gate != BETTY_GATE_NONE && has_y, has_u = a.u != nullptr;
  const int bytes_x = CH * 8 * G * (int)sizeof(TX), bytes_y = CH * 8 * G * (int)sizeof(TY);
  const uint32_t ring = shared_address(slots) + sub * (a.ahead + 1) * R * a.slot_bytes;
  auto gate_row = [&](int64_t r) { return row_at<TY>(a.g, a.per_gate == 1 ? r : (int64_t)((unsigned)r / a.per_gate), a.ldg); };
  auto fetch = [&](int64_t first, int slot) {
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        if (first + i >= n_rows) break;
        const int64_t r = row_of(first + i);
        const uint32_t p = ring + (slot * R + i) * a.slot_bytes;
        copy_row<CH>(p, row_at<TX>(a.x, r, a.ldx), w);
        if (has_y) copy_row<CH>(p + bytes_x, row_at<TY>(a.y, r, a.ldy), w);
        if (has_g) {
          if (a.gate_ahead) copy_row<CH>(p + bytes_x + bytes_y, gate_row(r), w);
          else fill_slot<CH, VEC>(p + bytes_x + bytes_y, gate_row(r), w);
        }
      }
      copies_commit();
    }
  };
  int half = 0, slot = 0;
  if (VEC)
    for (int i = 0; i < a.ahead; ++i) fetch(at + i * step, i);
  float wp[CH][8], ws[CH][8], bp[GENERAL ? CH : 1][8], bs[GENERAL ? CH : 1][8];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    float s[8];
    load8<VEC>(wp[c], a.params, c, w);
    load8<VEC>(ws[c], a.params + d, c, w);
    load8<VEC>(s, a.params + 2 * (int64_t)d, c, w);
    if (GENERAL) {
#pragma unroll
      for (int k = 0; k < 8; ++k) { bp[c][k] = 0.f; bs[c][k] = 0.f; }
      if (a.bias) {
        load8<VEC>(bp[c], a.params + 3 * (int64_t)d, c, w);
        load8<VEC>(bs[c], a.params + 4 * (int64_t)d, c, w);
      }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {      // the residual scale goes into the post-norm's parameters
      ws[c][k] *= s[k];
      if (GENERAL) bs[c][k] *= s[k];
    }
  }
  float mask[GENERAL ? CH : 1][8];      // 1 for columns of the row, 0 outside
  if (GENERAL)
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int k = 0; k < 8; ++k) mask[c][k] = inside<VEC>(w, c, k) ? 1.f : 0.f;
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
          for (int k = 0; k < 8; ++k) v[i][c][k] = fmaf(-mean, mask[c][k], v[i][c][k]);
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
  for (; at < n_rows; at += step) {
    uint32_t p = 0;
    const int64_t row = row_of(at);
    if constexpr (VEC) {
      fetch(at + a.ahead * step, slot == 0 ? a.ahead : slot - 1);
      copies_wait(a.ahead);
      p = ring + slot * R * a.slot_bytes;
      slot = slot == a.ahead ? 0 : slot + 1;
      if (w.shift)
#pragma unroll
        for (int i = 0; i < R; ++i) {
          drop_head<TX>(p + i * a.slot_bytes, w);
          if (has_y) drop_head<TY>(p + i * a.slot_bytes + bytes_x, w);
          if (has_g) drop_head<TY>(p + i * a.slot_bytes + bytes_x + bytes_y, w);
        }
    }
    float x[R][CH][8], y[R][CH][8], r[R];
    // rows past the last one hold whatever their slots hold; they take part in the sums and are not stored
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        if constexpr (VEC) {
          read_slot<TX>(x[i][c], p + i * a.slot_bytes, c, w);
          if (has_y) read_slot<TY>(y[i][c], p + i * a.slot_bytes + bytes_x, c, w);
        } else {
          load8<VEC>(x[i][c], row_at<TX>(a.x, row, a.ldx), c, w);
          if (has_y) load8<VEC>(y[i][c], row_at<TY>(a.y, row, a.ldy), c, w);
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
            if constexpr (VEC) read_slot<TY>(g, p + i * a.slot_bytes + bytes_x + bytes_y, c, w);
            else load8<VEC>(g, gate_row(row), c, w);
            if (a.gate == BETTY_GATE_SIGMOID)
#pragma unroll
              for (int k = 0; k < 8; ++k) g[k] = sigmoid_gate<TX>(g[k]);
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float z = GENERAL ? fmaf(y[i][c][k] * r[i], ws[c][k], bs[c][k]) : y[i][c][k] * r[i] * ws[c][k];
            x[i][c][k] = fmaf(g[k], z, x[i][c][k]);
          }
          if (R == 1 || at + i < n_rows) store8<VEC>(row_at<TX>(a.x_out, row + i * a.classes, a.ldxo), x[i][c], c, w);
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
          if (R == 1 || at + i < n_rows) store8<VEC>(row_at<TY>(a.u, row + i * a.classes, a.ldu), o, c, w);
        }
    }
  }
}

template <typename TX, typename TY, bool VEC, int CH, int R, bool GENERAL>
static betty_status launch_forward(cudaStream_t stream, const Args& a, const Layout& l) {
  static SmemLimit limit = {};
  if (l.smem > 40 * 1024) BETTY_TRY(ensure_dynamic_smem(k_forward<TX, TY, VEC, CH, R, GENERAL>, limit, l.smem));
  const int groups = l.threads / l.G;
  // thread groups: a multiple of the classes, so that every class is walked
  const int64_t per_class = ((a.rows + a.classes - 1) / a.classes + R - 1) / R, want = (per_class * a.classes + groups - 1) / groups;
  int64_t blocks = (int64_t)l.blocks_per_sm * current_sm_count();
  if (want < blocks) blocks = want;
  if (blocks * groups < a.classes) blocks = (a.classes + groups - 1) / groups;
  launch_pdl(k_forward<TX, TY, VEC, CH, R, GENERAL>, dim3((unsigned)blocks), dim3(l.threads), l.smem, stream, a);
  BETTY_LAUNCH_CHECK();
  return BETTY_OK;
}
// the wide kernel's chunks per thread and rows at a time: what 128 registers hold
static constexpr int FWD_CHUNKS = 2;
static constexpr int forward_batch(bool general) { return general ? 1 : 2; }
template <typename TX, typename TY, bool GENERAL>
static betty_status forward_layout(cudaStream_t stream, const Args& a, const Layout& l) {
  if (!l.vec) return launch_forward<TX, TY, false, 4, 1, GENERAL>(stream, a, l);
  if (l.wide) return launch_forward<TX, TY, true, FWD_CHUNKS, forward_batch(GENERAL), GENERAL>(stream, a, l);
  return l.chunks == 1 ? launch_forward<TX, TY, true, 1, 1, GENERAL>(stream, a, l) : launch_forward<TX, TY, true, 2, 1, GENERAL>(stream, a, l);
}
template <typename TX, typename TY>
static betty_status forward_typed(cudaStream_t stream, const Args& a, const Layout& l) {
  const bool general = a.bias || a.pre == BETTY_NORM_LAYER || a.post == BETTY_NORM_LAYER;
  return general ? forward_layout<TX, TY, true>(stream, a, l) : forward_layout<TX, TY, false>(stream, a, l);
}
betty_status forward(cudaStream_t stream, Args& a, int xd, int yd, int classes) {
  // a gate of several rows is fetched like the other streams where its rows start on 16-byte boundaries as theirs do
  a.gate_ahead = a.per_gate == 1 || (classes == 1 && a.ld8 == 0 && a.ldg % 16 == 0 && aligned16(a.g));
  const int ys = (a.y ? 1 : 0) + (a.y && a.gate != BETTY_GATE_NONE ? 1 : 0);
  const bool general = a.bias || a.pre == BETTY_NORM_LAYER || a.post == BETTY_NORM_LAYER;
  const Layout l = layout_of(a.d, a.rows, xd, yd, classes, {1, ys, FWD_CHUNKS, forward_batch(general), 0, 0});
  a.G = l.G; a.ahead = l.ahead; a.slot_bytes = l.slot_bytes; a.classes = l.vec ? classes : 1;
  if (xd == BETTY_F32 && yd == BETTY_F32) return forward_typed<float, float>(stream, a, l);
  if (xd == BETTY_F32 && yd == BETTY_BF16) return forward_typed<float, __nv_bfloat16>(stream, a, l);
  if (xd == BETTY_F32 && yd == BETTY_F16) return forward_typed<float, __half>(stream, a, l);
  if (xd == BETTY_BF16 && yd == BETTY_BF16) return forward_typed<__nv_bfloat16, __nv_bfloat16>(stream, a, l);
  return forward_typed<__half, __half>(stream, a, l);
}

// Many rows take the wide kernel (several chunks per thread: a row's fixed cost, its sums and addresses, is shared by more
// values); rows that would leave thread groups idle take one chunk per thread.  Rows that cannot be fetched ahead are read where they
// are used, four chunks per thread: those without a common shift, those of which one does not fit the shared memory, and, backward,
// fp32 rows of 257 to 512 values with a gate and layer norms or biases (with a gate to each row of 7169 to 8192, too): the blocks
// that the group size gives an SM leave no room for two rows and the coefficients.  Wide rows of which only one fits are fetched
// when it is their turn (backward, a gate to each row, 4096 rows, single launches: 8192 bf16 values 116 us, read where they are used
// 501; 6144 fp32 values 282 and 490).
Layout layout_of(int64_t d, int64_t rows, int xd, int yd, int classes, const Needs& n) {
  const int bx = xd == BETTY_F32 ? 4 : 2, by = yd == BETTY_F32 ? 4 : 2, sms = current_sm_count();
  const int64_t span = classes > 1 ? d + 7 : d;              // columns with the head of a shifted row
  for (int attempt = classes > 0 ? 0 : 3; ; ++attempt) {     // wide, one chunk per thread, two, not fetched ahead
    Layout l = {};
    l.vec = attempt < 3;
    l.wide = attempt == 0;
    l.chunks = attempt == 0 ? n.wide_chunks : (attempt == 3 ? MAX_CH : attempt);
    const int batch = attempt == 0 ? n.batch : 1;
    const int64_t need = l.vec ? span : d;
    l.G = 32;
    while (l.G < MAX_G && (int64_t)l.G * 8 * l.chunks < need) l.G += 32;
    if ((int64_t)l.G * 8 * l.chunks < need) continue;
    l.threads = l.G == 32 ? SMALL_THREADS : l.G;
    const int groups = l.threads / l.G;
    l.blocks_per_sm = MAX_G / l.threads;
    l.slot_bytes = l.chunks * 8 * l.G * (n.streams_x * bx + n.streams_y * by);
    const size_t acc = (size_t)((l.vec ? n.kept_arrays : 0) + n.sum_arrays) * groups * l.chunks * 8 * l.G * sizeof(float);
    if (!l.vec) {
      l.smem = acc;
      l.slot_bytes = 0;
      return l;
    }
    if (l.wide && span <= (int64_t)MAX_G * 8 && rows < (int64_t)2 * batch * groups * l.blocks_per_sm * sms) continue;
    // the last 5 KB (left to L1 elsewhere) where a row would not fit without them: 4096 x 8192 fp32 RMS backward 364 us, read
    // where it is used 595
    const int64_t most = (attempt == 2 ? 227 : 222) * 1024;
    const int64_t slot = (int64_t)l.slot_bytes * groups * batch, budget = most / l.blocks_per_sm - 2048 - (int64_t)acc;
    l.ahead = (int)(budget / slot) - 1;
    if (l.ahead < (attempt == 2 ? 0 : 1)) continue;
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
// The matrices of a call: `classes` becomes 0 when their rows do not all start at the same shift (see block_norm.cuh), else
// the period of the shifts.
struct Rows { int64_t ld; int classes; };      // ld: modulo 8, or -1 before the first matrix
static inline int classes_of(int64_t ld8) { return ld8 == 0 ? 1 : (ld8 == 4 ? 2 : (ld8 % 2 == 0 ? 4 : 8)); }
static betty_status check_matrix(const void* p, int64_t ld, int64_t rows, int64_t d, int dtype, Rows& r) {
  if (!p) return BETTY_OK;
  if (rows > 1 && ld < d) return BETTY_ERR_SHAPE;
  if (rows > 1 && ld >= (1 << 30)) return BETTY_ERR_UNSUPPORTED;      // row addresses take 32-bit strides in bytes
  if ((uintptr_t)p % size_of(dtype)) return BETTY_ERR_ALIGNMENT;
  if (!aligned16(p)) r.classes = 0;
  if (rows > 1) {
    if (r.ld >= 0 && r.ld != (ld & 7)) r.classes = 0;
    r.ld = ld & 7;
    if (r.classes) r.classes = classes_of(r.ld);
  }
  return BETTY_OK;
}
// a gate that several rows share is read and written value by value: its rows need no common shift
static betty_status check_gate(const betty_block_norm_cfg* c, const void* p, int64_t ld, int64_t rows, Rows& r) {
  Rows own = r;
  BETTY_TRY(check_matrix(p, ld, (rows + c->rows_per_gate - 1) / c->rows_per_gate, c->d, c->y_dtype, c->rows_per_gate == 1 ? r : own));
  return BETTY_OK;
}
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
  Rows r = {-1, 1};
  BETTY_TRY(check_matrix(x, ldx, rows, d, cfg->x_dtype, r));
  BETTY_TRY(check_matrix(y, ldy, rows, d, cfg->y_dtype, r));
  if (y) BETTY_TRY(check_matrix(x_out, ldxo, rows, d, cfg->x_dtype, r));
  if (y && cfg->gate != BETTY_GATE_NONE)
    BETTY_TRY(check_gate(cfg, gate, ldg, rows, r));
  BETTY_TRY(check_matrix(u, ldu, rows, d, cfg->y_dtype, r));
  Args a = {};
  common_args(a, cfg, rows, params);
  const uint32_t bx = (uint32_t)size_of(cfg->x_dtype), by = (uint32_t)size_of(cfg->y_dtype);
  a.x = x; a.ldx = (uint32_t)ldx * bx; a.y = y; a.ldy = (uint32_t)ldy * by; a.g = gate; a.ldg = (uint32_t)ldg * by;
  a.x_out = x_out; a.ldxo = (uint32_t)ldxo * bx; a.u = u; a.ldu = (uint32_t)ldu * by;
  a.ld8 = r.ld > 0 ? (int)r.ld : 0;
  return forward((cudaStream_t)stream, a, cfg->x_dtype, cfg->y_dtype, r.classes);
}

extern "C" betty_status betty_block_norm_workspace_size_for(const betty_block_norm_cfg* cfg, int64_t rows, int32_t any_layout, size_t* bytes) {
  if (!bytes) return BETTY_ERR_INVALID_ARG;
  BETTY_TRY(check_cfg(cfg, rows));
  const bool shared = cfg->gate != BETTY_GATE_NONE && cfg->rows_per_gate > 1;
  int64_t floats = 0;
  // whatever the matrices' types will be, and their addresses: none (0: not at one shift, 1: one row) or those of their own width
  for (int classes : {0, 1, 2, 4, 8}) {
    if (!any_layout && classes > 1 && classes != classes_of(cfg->d & 7)) continue;
    for (int xd : {BETTY_F32, BETTY_BF16})
      for (int yd : {BETTY_F32, BETTY_BF16})
        for (int64_t r : {rows, (int64_t)0}) {       // fewer rows may take the other layout, of more and smaller blocks
          const Layout l = backward_layout(cfg, r, xd, yd, classes);
          int blocks, shares;
          const int used = l.vec ? classes : 1;
          backward_grid(rows, l, used, blocks, shares);
          const int64_t sums = shared ? used * gate_sums_of(rows, cfg->rows_per_gate, used, shares).rows : 0;
          const int64_t n = ((int64_t)blocks * quantities(cfg) + sums) * cfg->d;
          if (n > floats) floats = n;
        }
  }
  *bytes = sizeof(StatusBlock) + 2 * 256 + (size_t)floats * sizeof(float);
  return BETTY_OK;
}
extern "C" betty_status betty_block_norm_workspace_size(const betty_block_norm_cfg* cfg, int64_t rows, size_t* bytes) {
  return betty_block_norm_workspace_size_for(cfg, rows, 1, bytes);
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
  const bool gated = rows > 0 && y && cfg->gate != BETTY_GATE_NONE;      // without rows there is no gate row to read either
  Args a = {};
  Rows r = {-1, 1};
  if (rows > 0) {
    if ((!x_out && du) || (!du && !dx_out) || (!y && !du) || !dx || (y && !dy) || (gated && (!gate || !dgate))) return BETTY_ERR_INVALID_ARG;
    BETTY_TRY(check_matrix(x_out, ldxo, rows, d, cfg->x_dtype, r));
    BETTY_TRY(check_matrix(y, ldy, rows, d, cfg->y_dtype, r));
    BETTY_TRY(check_matrix(du, lddu, rows, d, cfg->y_dtype, r));
    BETTY_TRY(check_matrix(dx_out, lddxo, rows, d, cfg->x_dtype, r));
    BETTY_TRY(check_matrix(dx, lddx, rows, d, cfg->x_dtype, r));
    if (y) BETTY_TRY(check_matrix(dy, lddy, rows, d, cfg->y_dtype, r));
    if (gated) {
      BETTY_TRY(check_gate(cfg, gate, ldg, rows, r));
      BETTY_TRY(check_gate(cfg, dgate, lddg, rows, r));
    }
  }
  common_args(a, cfg, rows, params);
  if (!gated) a.gate = BETTY_GATE_NONE;
  const uint32_t bx = (uint32_t)size_of(cfg->x_dtype), by = (uint32_t)size_of(cfg->y_dtype);
  a.x = x_out; a.ldx = (uint32_t)ldxo * bx; a.y = y; a.ldy = (uint32_t)ldy * by; a.g = gate; a.ldg = (uint32_t)ldg * by;
  a.du = du; a.lddu = (uint32_t)lddu * by; a.dxo = dx_out; a.lddxo = (uint32_t)lddxo * bx;
  a.dx = dx; a.lddx = (uint32_t)lddx * bx; a.dy = dy; a.lddy = (uint32_t)lddy * by; a.dg = dgate; a.lddg = (uint32_t)lddg * by;
  Arena arena(ws, ws_bytes);
  const Layout l = backward_layout(cfg, rows, cfg->x_dtype, cfg->y_dtype, r.classes);
  int blocks;
  a.classes = l.vec ? r.classes : 1;
  a.ld8 = r.ld > 0 ? (int)r.ld : 0;
  backward_grid(rows, l, a.classes, blocks, a.shares);
  a.col_partials = arena.alloc<float>((size_t)blocks * quantities(cfg) * d);
  if (gated && cfg->rows_per_gate > 1) {
    a.gate_sums = gate_sums_of(rows, cfg->rows_per_gate, a.classes, a.shares);
    a.gate_partials = arena.alloc<float>((size_t)(a.classes * a.gate_sums.rows) * d);
  }
  if (arena.overflow) return BETTY_ERR_WORKSPACE;
  return backward((cudaStream_t)stream, a, l, cfg->x_dtype, cfg->y_dtype, dparams);
}
