// Backward pass of the block norm (see block_norm.cuh).  With n = N_pre(x') = r * (x' - mean), m = N_post(y) = q * (y - mean),
// dn = du * w_pre and <.> the mean over a row:
//
//   dX = dx' + r * (dn - n <dn n> - [layer] <dn>)                      the gradient of x (and of the whole sum)
//   dm = dX * s * a * w_post,   dy = q * (dm - m <dm m> - [layer] <dm>)
//   dg = dX * s * (m w_post + b_post) * a'(g)                          summed over the rows that share the gate
//   dw_pre = sum du n,  db_pre = sum du,  dw_post = s A,  db_post = s B,  ds = w_post A + b_post B,
//   A = sum over rows of dX a m,  B = sum over rows of dX a
//
// Both norms' statistics are taken again from x' and y, which have to be read anyway: nothing is kept from the forward pass.
#include <type_traits>
#include "block_norm.cuh"

namespace betty {
namespace blocknorm {

// First row of a walker's share; the shares are contiguous and differ by at most one row.
__host__ __device__ __forceinline__ int64_t share_start(int64_t w, int64_t rows, int64_t walkers) { return w * rows / walkers; }
__device__ __forceinline__ int64_t walker_of(int64_t row, int64_t rows, int64_t walkers) { return ((row + 1) * walkers - 1) / rows; }

// Each walker (thread group) takes a contiguous share of the rows, so that the column sums (parameter gradients, gates of
// several rows) stay in its registers; it writes them once, and k_backward_sums adds the walkers' sums in order.
// Per row: the norms' sums over the fetched values, then dX (and with it everything that hangs off dm), then dy.
template <typename TX, typename TY, int GR, bool PIPE, int CH, bool GENERAL>
__global__ void __launch_bounds__(MAX_G, 1) k_backward(const Args a) {
  __shared__ float red[2 * RED_VALUES * 16];
  extern __shared__ __align__(16) char slots[];      // fetched rows; G = 32: at the end the warps' column sums
  pdl_enter();
  const int G = a.G, d = a.d, t = threadIdx.x & (G - 1), sub = threadIdx.x / G;
  const int64_t walker = (int64_t)blockIdx.x * (blockDim.x / G) + sub;
  const int64_t first = share_start(walker, a.rows, a.walkers), last = share_start(walker + 1, a.rows, a.walkers);
  const bool has_y = a.y != nullptr, has_g = a.gate != BETTY_GATE_NONE, has_u = a.du != nullptr, has_o = a.dxo != nullptr;
  const bool pre_layer = GENERAL && a.pre == BETTY_NORM_LAYER && has_u, post_layer = GENERAL && a.post == BETTY_NORM_LAYER && has_y;
  const bool shared_gate = has_g && a.per_gate > 1;
  const float* w_pre = a.params;
  const float* w_post = a.params + d;
  const float* s_res = a.params + 2 * (int64_t)d;
  const float* b_post = a.params + 4 * (int64_t)d;
  const int bx = CH * 8 * G * (int)sizeof(TX), by = CH * 8 * G * (int)sizeof(TY);
  const int at_o = bx, at_y = 2 * bx, at_u = 2 * bx + by, at_g = 2 * bx + 2 * by;
  char* ring = slots + (size_t)sub * (a.ahead + 1) * a.slot_bytes;
  auto gate_row = [&](int64_t r) { return (const TY*)a.g + (int64_t)((unsigned)r / a.per_gate) * a.ldg; };
  auto fetch = [&](int64_t r, int slot) {
    if constexpr (PIPE) {
      if (r < last) {
        char* p = ring + slot * a.slot_bytes;
        if (has_u) {
          copy_row<GR, CH>(p, (const TX*)a.x + r * a.ldx, t, G, d);
          copy_row<GR, CH>(p + at_u, (const TY*)a.du + r * a.lddu, t, G, d);
        }
        if (has_o) copy_row<GR, CH>(p + at_o, (const TX*)a.dxo + r * a.lddxo, t, G, d);
        if (has_y) copy_row<GR, CH>(p + at_y, (const TY*)a.y + r * a.ldy, t, G, d);
        if (has_g) copy_row<GR, CH>(p + at_g, gate_row(r), t, G, d);
      }
      copies_commit();
    }
  };
  // one chunk of a stream of the present row
  const char* p = nullptr;
  auto get = [&](auto* base, int64_t row, int64_t ld, int at, int c, float (&v)[8]) {
    typedef typename std::remove_const<typename std::remove_pointer<decltype(base)>::type>::type T;
    if constexpr (PIPE) read_slot<GR, T>(v, p + at, c, t, G, d);
    else load8<GR, T>(v, base + row * ld, c, t, G, d);
  };
  // parameters of one chunk: kept in registers where a thread holds one chunk, else read again (they stay in L1)
  constexpr int KEEP = CH == 1 ? 1 : 0;
  float kp[KEEP ? 8 : 1], kws[KEEP ? 8 : 1];
  auto param_pre = [&](int c, float (&v)[8]) {
    if constexpr (KEEP) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = kp[k];
    } else load_param8<GR>(v, w_pre, c, t, G, d);
  };
  auto param_post = [&](int c, float (&v)[8]) {      // w_post * s
    if constexpr (KEEP) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = kws[k];
    } else {
      float s[8];
      load_param8<GR>(v, w_post, c, t, G, d);
      load_param8<GR>(s, s_res, c, t, G, d);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] *= s[k];
    }
  };
  int half = 0, slot = 0;
  if (PIPE)
    for (int i = 0; i < a.ahead; ++i) fetch(first + i, i);
  if constexpr (KEEP) {
    float s[8];
    load_param8<GR>(kp, w_pre, 0, t, G, d);
    load_param8<GR>(kws, w_post, 0, t, G, d);
    load_param8<GR>(s, s_res, 0, t, G, d);
#pragma unroll
    for (int k = 0; k < 8; ++k) kws[k] *= s[k];
  }
  float accC[CH][8], accA[CH][8], accD[GENERAL ? CH : 1][8], accB[GENERAL ? CH : 1][8], accG[CH][8];
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      accC[c][k] = 0.f; accA[c][k] = 0.f; accG[c][k] = 0.f;
      if (GENERAL) { accD[c][k] = 0.f; accB[c][k] = 0.f; }
    }
  for (int64_t row = first; row < last; ++row) {
    if (PIPE) {
      fetch(row + a.ahead, slot == 0 ? a.ahead : slot - 1);
      copies_wait(a.ahead);
      p = ring + slot * a.slot_bytes;
      slot = slot == a.ahead ? 0 : slot + 1;
    }
    const TX* xs = (const TX*)a.x;
    const TX* os = (const TX*)a.dxo;
    const TY* ys = (const TY*)a.y;
    const TY* us = (const TY*)a.du;
    float mean_dn = 0.f, mx = 0.f, my = 0.f;
    if (pre_layer || post_layer) {
      float v[3] = {0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float x[8], y[8], du[8], w[8];
        if (pre_layer) {
          get(xs, row, a.ldx, 0, c, x);
          get(us, row, a.lddu, at_u, c, du);
          param_pre(c, w);
#pragma unroll
          for (int k = 0; k < 8; ++k) { v[0] += x[k]; v[2] = fmaf(du[k], w[k], v[2]); }
        }
        if (post_layer) {
          get(ys, row, a.ldy, at_y, c, y);
#pragma unroll
          for (int k = 0; k < 8; ++k) v[1] += y[k];
        }
      }
      row_sums<3>(v, red, half, G, t);
      if (pre_layer) { mx = v[0] * a.inv_d; mean_dn = v[2] * a.inv_d; }
      if (post_layer) my = v[1] * a.inv_d;
    }
    float r = 1.f, q = 1.f, proj = 0.f;
    {
      float v[3] = {0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        if (has_u) {
          float x[8], du[8], w[8];
          get(xs, row, a.ldx, 0, c, x);
          get(us, row, a.lddu, at_u, c, du);
          param_pre(c, w);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            if (GENERAL) x[k] = column<GR>(c, k, t, G) < d ? x[k] - mx : 0.f;
            v[0] = fmaf(x[k], x[k], v[0]);
            v[1] = fmaf(du[k] * w[k], x[k], v[1]);
          }
        }
        if (has_y) {
          float y[8];
          get(ys, row, a.ldy, at_y, c, y);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            if (GENERAL) y[k] = column<GR>(c, k, t, G) < d ? y[k] - my : 0.f;
            v[2] = fmaf(y[k], y[k], v[2]);
          }
        }
      }
      row_sums<3>(v, red, half, G, t);
      if (a.pre != BETTY_NORM_NONE && has_u) {
        r = rsqrtf(fmaf(v[0], a.inv_d, a.eps));
        proj = r * v[1] * a.inv_d;
      }
      if (a.post != BETTY_NORM_NONE && has_y) q = rsqrtf(fmaf(v[2], a.inv_d, a.eps));
    }
    TX* dx = (TX*)a.dx + row * a.lddx;
    float v[2] = {0.f, 0.f};
    float m[CH][8], dm[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float dX[8];
      if (has_o) get(os, row, a.lddxo, at_o, c, dX);
      else
#pragma unroll
        for (int k = 0; k < 8; ++k) dX[k] = 0.f;
      if (has_u) {
        float x[8], du[8], w[8];
        get(xs, row, a.ldx, 0, c, x);
        get(us, row, a.lddu, at_u, c, du);
        param_pre(c, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float n = (GENERAL ? x[k] - mx : x[k]) * r;
          accC[c][k] = fmaf(du[k], n, accC[c][k]);
          if (GENERAL) accD[c][k] += du[k];
          float dn = fmaf(-n, proj, du[k] * w[k]);
          if (GENERAL) dn -= mean_dn;
          dX[k] = fmaf(r, dn, dX[k]);
        }
      }
      store8<GR>(dx, dX, c, t, G, d);
      if (!has_y) continue;
      float ws[8], g[8], b[8], y[8];
      param_post(c, ws);
      get(ys, row, a.ldy, at_y, c, y);
      if (has_g) get((const TY*)a.g, (int64_t)((unsigned)row / a.per_gate), a.ldg, at_g, c, g);
      if (GENERAL && a.bias) {
        float s[8];
        load_param8<GR>(b, b_post, c, t, G, d);
        load_param8<GR>(s, s_res, c, t, G, d);
#pragma unroll
        for (int k = 0; k < 8; ++k) b[k] *= s[k];
      }
      float dg[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float mk = (GENERAL ? (column<GR>(c, k, t, G) < d ? y[k] - my : 0.f) : y[k]) * q;
        float act = 1.f, slope = 1.f;
        if (a.gate == BETTY_GATE_LINEAR) act = g[k];
        if (a.gate == BETTY_GATE_SIGMOID) { act = sigmoid_f(g[k]); slope = act * (1.f - act); }
        const float base = dX[k] * act, dmk = base * ws[k];
        accA[c][k] = fmaf(base, mk, accA[c][k]);
        float z = mk * ws[k];
        if (GENERAL) {
          accB[c][k] += base;
          if (a.bias) z += b[k];
        }
        dg[k] = dX[k] * z * slope;
        accG[c][k] += dg[k];
        v[0] = fmaf(dmk, mk, v[0]);
        v[1] += dmk;
        m[c][k] = mk;
        dm[c][k] = dmk;
      }
      if (has_g && !shared_gate) store8<GR>((TY*)a.dg + row * a.lddg, dg, c, t, G, d);
    }
    if (!has_y) continue;
    if (a.post != BETTY_NORM_NONE) row_sums<2>(v, red, half, G, t);
    const float pm = a.post != BETTY_NORM_NONE ? v[0] * a.inv_d : 0.f, mean_dm = post_layer ? v[1] * a.inv_d : 0.f;
    TY* dy = (TY*)a.dy + row * a.lddy;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float o[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        o[k] = fmaf(-m[c][k], pm, dm[c][k]);
        if (GENERAL) o[k] -= mean_dm;
        o[k] *= q;
      }
      store8<GR>(dy, o, c, t, G, d);
    }
    if (shared_gate) {
      const unsigned gate = (unsigned)row / a.per_gate;
      const int64_t g0 = (int64_t)gate * a.per_gate;
      const int64_t g1 = g0 + a.per_gate < a.rows ? g0 + a.per_gate : a.rows;
      if (row + 1 == g1 || row + 1 == last) {
        const bool whole = g0 >= first && g1 <= last;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          if (whole) store8<GR>((TY*)a.dg + gate * a.lddg, accG[c], c, t, G, d);
          else store8<GR>(a.gate_partials + (walker + gate) * d, accG[c], c, t, G, d);
#pragma unroll
          for (int k = 0; k < 8; ++k) accG[c][k] = 0.f;
        }
      }
    }
  }
  const int nq = a.bias ? 4 : 2;
  float* out = a.col_partials + (int64_t)blockIdx.x * nq * d;
  if (G > 32) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      store8<GR>(out, accC[c], c, t, G, d);
      store8<GR>(out + d, accA[c], c, t, G, d);
      if (GENERAL && a.bias) {
        store8<GR>(out + 2 * (int64_t)d, accD[c], c, t, G, d);
        store8<GR>(out + 3 * (int64_t)d, accB[c], c, t, G, d);
      }
    }
  } else {                                    // a warp per walker: the block's warps are added in order through shared memory
    float* combine = (float*)slots;
    constexpr int W = CH * 256;               // columns a warp can hold
    const int warps = blockDim.x >> 5;
    for (int qn = 0; qn < nq; ++qn) {
      __syncthreads();
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          float s = qn == 0 ? accC[c][k] : accA[c][k];
          if (GENERAL && qn >= 2) s = qn == 2 ? accD[c][k] : accB[c][k];
          combine[sub * W + column<GR>(c, k, t, 32)] = s;
        }
      __syncthreads();
      for (int j = threadIdx.x; j < d; j += blockDim.x) {
        float s = 0.f;
        for (int w = 0; w < warps; ++w) s += combine[w * W + j];
        out[(int64_t)qn * d + j] = s;
      }
    }
  }
}

// Adds the blocks' column sums and forms the parameter gradients (the first param_blocks blocks: 32 columns each, eight
// slices of the list added in a fixed order), then the gates whose rows lie in several walkers' shares (256 columns each).
template <typename TY>
__global__ void __launch_bounds__(256) k_backward_sums(const Args a, int blocks, int param_blocks, float* __restrict__ dparams) {
  __shared__ float part[4][8][32];
  pdl_enter();
  const int d = a.d;
  if ((int)blockIdx.x < param_blocks) {
    const int j = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5, nq = a.bias ? 4 : 2;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (j < d)
#pragma unroll 4
      for (int b = slice; b < blocks; b += 8) {
        const float* p = a.col_partials + (int64_t)b * nq * d + j;
        v[0] += p[0];
        v[1] += p[d];
        if (nq == 4) { v[2] += p[2 * (int64_t)d]; v[3] += p[3 * (int64_t)d]; }
      }
#pragma unroll
    for (int i = 0; i < 4; ++i) part[i][slice][threadIdx.x & 31] = v[i];
    __syncthreads();
    if (slice == 0 && j < d) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = 0.f;
#pragma unroll
        for (int s = 0; s < 8; ++s) v[i] += part[i][s][threadIdx.x];
      }
      const float w = a.params[d + j], s = a.params[2 * (int64_t)d + j];
      dparams[j] = v[0];
      dparams[d + j] = s * v[1];
      float ds = w * v[1];
      if (nq == 4) {
        ds = fmaf(a.params[4 * (int64_t)d + j], v[3], ds);
        dparams[3 * (int64_t)d + j] = v[2];
        dparams[4 * (int64_t)d + j] = s * v[3];
      }
      dparams[2 * (int64_t)d + j] = ds;
    }
    return;
  }
  const int col_blocks = (d + 255) / 256;
  const int item = (blockIdx.x - param_blocks) / col_blocks, j = ((blockIdx.x - param_blocks) % col_blocks) * 256 + threadIdx.x;
  const int64_t gates = (a.rows + a.per_gate - 1) / a.per_gate;
  int64_t gate = item;
  if (gates >= a.walkers) {      // more gates than shares: only the ones cut by the start of share item + 1 are open
    const int64_t cut = share_start(item + 1, a.rows, a.walkers);
    gate = cut / a.per_gate;
    const int64_t g0 = gate * a.per_gate;
    if (g0 == cut || walker_of(g0, a.rows, a.walkers) != item) return;
  }
  const int64_t g0 = gate * a.per_gate, g1 = g0 + a.per_gate < a.rows ? g0 + a.per_gate : a.rows;
  const int64_t lo = walker_of(g0, a.rows, a.walkers), hi = walker_of(g1 - 1, a.rows, a.walkers);
  if (lo == hi || j >= d) return;
  float s = 0.f;
#pragma unroll 4
  for (int64_t w = lo; w <= hi; ++w)
    if (share_start(w, a.rows, a.walkers) < share_start(w + 1, a.rows, a.walkers)) s += a.gate_partials[(w + gate) * d + j];
  ((TY*)a.dg)[gate * a.lddg + j] = from_f<TY>(s);
}

int backward_blocks(int64_t rows, const Layout& l) {
  const int per_block = l.threads / l.G;
  const int64_t want = (rows + per_block - 1) / per_block, most = (int64_t)current_sm_count() * l.blocks_per_sm;
  return (int)(want < 1 ? 1 : (want < most ? want : most));
}
Layout backward_layout(int64_t d, int xd, int yd, int granule) {
  Layout l = layout_of(d, xd, yd, granule, 2, 3, 512, 1);
  const size_t combine = l.G == 32 ? (size_t)(l.threads / 32) * l.chunks * 256 * sizeof(float) : 0;
  if (l.smem < combine) l.smem = combine;
  return l;
}

template <typename TX, typename TY, int GR, bool PIPE, int CH, bool GENERAL>
static betty_status launch_backward(cudaStream_t stream, const Args& a, const Layout& l, float* dparams) {
  static SmemLimit limit = {};
  if (l.smem > 40 * 1024) BETTY_TRY(ensure_dynamic_smem(k_backward<TX, TY, GR, PIPE, CH, GENERAL>, limit, l.smem));
  const int blocks = a.walkers / (l.threads / l.G);
  launch_pdl(k_backward<TX, TY, GR, PIPE, CH, GENERAL>, dim3(blocks), dim3(l.threads), l.smem, stream, a);
  BETTY_LAUNCH_CHECK();
  const int param_blocks = (a.d + 31) / 32;
  int64_t items = 0;
  if (a.gate_partials && a.rows > 0) {
    const int64_t gates = (a.rows + a.per_gate - 1) / a.per_gate;
    items = gates < a.walkers ? gates : a.walkers - 1;
  }
  launch_pdl(k_backward_sums<TY>, dim3((unsigned)(param_blocks + items * ((a.d + 255) / 256))), dim3(256), 0, stream, a, blocks, param_blocks,
             dparams);
  BETTY_LAUNCH_CHECK();
  return BETTY_OK;
}
template <typename TX, typename TY, bool GENERAL>
static betty_status backward_shape(cudaStream_t stream, const Args& a, const Layout& l, float* dparams) {
  if (l.granule == 8) {
    if (!l.ahead) return launch_backward<TX, TY, 8, false, 4, GENERAL>(stream, a, l, dparams);
    return l.chunks == 1 ? launch_backward<TX, TY, 8, true, 1, GENERAL>(stream, a, l, dparams)
                         : launch_backward<TX, TY, 8, true, 2, GENERAL>(stream, a, l, dparams);
  }
  if constexpr (sizeof(TY) == 4) {
    if (l.ahead) return launch_backward<TX, TY, 1, true, 1, GENERAL>(stream, a, l, dparams);
  } else {
    if (l.ahead) return launch_backward<TX, TY, 2, true, 1, GENERAL>(stream, a, l, dparams);
    if (l.chunks == 1) return launch_backward<TX, TY, 1, false, 1, GENERAL>(stream, a, l, dparams);
  }
  return launch_backward<TX, TY, 1, false, 4, GENERAL>(stream, a, l, dparams);
}
template <typename TX, typename TY>
static betty_status backward_typed(cudaStream_t stream, const Args& a, const Layout& l, float* dparams) {
  const bool general = a.bias || a.pre == BETTY_NORM_LAYER || a.post == BETTY_NORM_LAYER;
  return general ? backward_shape<TX, TY, true>(stream, a, l, dparams) : backward_shape<TX, TY, false>(stream, a, l, dparams);
}
betty_status backward(cudaStream_t stream, Args& a, const Layout& l, int xd, int yd, float* dparams) {
  a.G = l.G; a.ahead = l.ahead; a.slot_bytes = l.slot_bytes;
  if (xd == BETTY_F32 && yd == BETTY_F32) return backward_typed<float, float>(stream, a, l, dparams);
  if (xd == BETTY_F32 && yd == BETTY_BF16) return backward_typed<float, __nv_bfloat16>(stream, a, l, dparams);
  if (xd == BETTY_F32 && yd == BETTY_F16) return backward_typed<float, __half>(stream, a, l, dparams);
  if (xd == BETTY_BF16 && yd == BETTY_BF16) return backward_typed<__nv_bfloat16, __nv_bfloat16>(stream, a, l, dparams);
  return backward_typed<__half, __half>(stream, a, l, dparams);
}

}  // namespace blocknorm
}  // namespace betty
