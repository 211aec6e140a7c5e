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
#include "block_norm.cuh"

namespace betty {
namespace blocknorm {

// First row of a walker's share; the shares are contiguous and differ by at most one row.
__host__ __device__ __forceinline__ int64_t share_start(int64_t w, int64_t rows, int64_t walkers) { return w * rows / walkers; }
__device__ __forceinline__ int64_t walker_of(int64_t row, int64_t rows, int64_t walkers) { return ((row + 1) * walkers - 1) / rows; }

// Each walker (thread group) takes a contiguous share of the rows, so that the column sums (parameter gradients, gates of
// several rows) stay in its registers; it writes them once, and k_backward_sums adds the walkers' sums in order.
template <typename TX, typename TY, bool ALIGNED, int CH, bool GENERAL>
__global__ void __launch_bounds__(MAX_G) k_backward(const Args a) {
  __shared__ float red[2 * RED_VALUES * 32];
  extern __shared__ float combine[];          // G = 32: the warps' column sums
  pdl_enter();
  const int G = a.G, d = a.d, t = threadIdx.x & (G - 1);
  const int64_t walker = (int64_t)blockIdx.x * (blockDim.x / G) + threadIdx.x / G;
  const int64_t first = share_start(walker, a.rows, a.walkers), last = share_start(walker + 1, a.rows, a.walkers);
  const bool has_y = a.y != nullptr, has_g = a.gate != BETTY_GATE_NONE, has_u = a.du != nullptr, has_o = a.dxo != nullptr;
  const bool pre_layer = GENERAL && a.pre == BETTY_NORM_LAYER && has_u, post_layer = GENERAL && a.post == BETTY_NORM_LAYER && has_y;
  const bool shared_gate = has_g && a.per_gate > 1;
  const float* w_pre = a.params;
  const float* w_post = a.params + d;
  const float* s_res = a.params + 2 * (int64_t)d;
  const float* b_post = a.params + 4 * (int64_t)d;
  int half = 0;
  float accC[CH][8], accA[CH][8], accD[GENERAL ? CH : 1][8], accB[GENERAL ? CH : 1][8], accG[CH][8];
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      accC[c][k] = 0.f; accA[c][k] = 0.f; accG[c][k] = 0.f;
      if (GENERAL) { accD[c][k] = 0.f; accB[c][k] = 0.f; }
    }
  Raw8<TX> xr[CH], orr[CH];
  Raw8<TY> yr[CH], gr[CH], ur[CH];
  auto request = [&](int64_t r) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if (has_u) {
        load8<ALIGNED>(xr[c], (const TX*)a.x + r * a.ldx, c, t, G, d);
        load8<ALIGNED>(ur[c], (const TY*)a.du + r * a.lddu, c, t, G, d);
      }
      if (has_o) load8<ALIGNED>(orr[c], (const TX*)a.dxo + r * a.lddxo, c, t, G, d);
      if (has_y) load8<ALIGNED>(yr[c], (const TY*)a.y + r * a.ldy, c, t, G, d);
      if (has_g) load8<ALIGNED>(gr[c], (const TY*)a.g + (int64_t)((unsigned)r / a.per_gate) * a.ldg, c, t, G, d);
    }
  };
  if (first < last) request(first);
  for (int64_t row = first; row < last; ++row) {
    float x[CH][8], y[CH][8], du[CH][8], g[CH][8], dX[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[c][k] = has_u ? to_f(xr[c].v[k]) : 0.f;
        du[c][k] = has_u ? to_f(ur[c].v[k]) : 0.f;
        dX[c][k] = has_o ? to_f(orr[c].v[k]) : 0.f;
        y[c][k] = has_y ? to_f(yr[c].v[k]) : 0.f;
        g[c][k] = has_g ? to_f(gr[c].v[k]) : 0.f;
      }
    if (row + 1 < last) request(row + 1);
    float mean_dn = 0.f;
    if (pre_layer || post_layer) {
      float v[3] = {0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float w[8];
        load_param8<ALIGNED>(w, w_pre, c, t, G, d);
#pragma unroll
        for (int k = 0; k < 8; ++k) { v[0] += x[c][k]; v[1] += y[c][k]; v[2] = fmaf(du[c][k], w[k], v[2]); }
      }
      row_sums<3>(v, red, half, G, t);
      const float mx = pre_layer ? v[0] * a.inv_d : 0.f, my = post_layer ? v[1] * a.inv_d : 0.f;
      mean_dn = pre_layer ? v[2] * a.inv_d : 0.f;
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const bool in = column<ALIGNED>(c, k, t, G) < d;
          x[c][k] = in ? x[c][k] - mx : 0.f;
          y[c][k] = in ? y[c][k] - my : 0.f;
        }
    }
    float r = 1.f, q = 1.f, proj = 0.f;
    {
      float v[3] = {0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float w[8];
        load_param8<ALIGNED>(w, w_pre, c, t, G, d);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          v[0] = fmaf(x[c][k], x[c][k], v[0]);
          v[1] = fmaf(du[c][k] * w[k], x[c][k], v[1]);
          v[2] = fmaf(y[c][k], y[c][k], v[2]);
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
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float w[8];
      load_param8<ALIGNED>(w, w_pre, c, t, G, d);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float n = x[c][k] * r;
        accC[c][k] = fmaf(du[c][k], n, accC[c][k]);
        if (GENERAL) accD[c][k] += du[c][k];
        dX[c][k] = fmaf(r, du[c][k] * w[k] - n * proj - mean_dn, dX[c][k]);
      }
      store8<ALIGNED>(dx, dX[c], c, t, G, d);
    }
    if (!has_y) continue;
    float v[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float w[8], s[8], b[8], dg[8];
      load_param8<ALIGNED>(w, w_post, c, t, G, d);
      load_param8<ALIGNED>(s, s_res, c, t, G, d);
      if (GENERAL && a.bias) load_param8<ALIGNED>(b, b_post, c, t, G, d);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float m = y[c][k] * q;
        float act = 1.f, slope = 1.f;
        if (a.gate == BETTY_GATE_LINEAR) act = g[c][k];
        if (a.gate == BETTY_GATE_SIGMOID) { act = sigmoid_f(g[c][k]); slope = act * (1.f - act); }
        const float base = dX[c][k] * act, ws = w[k] * s[k];
        accA[c][k] = fmaf(base, m, accA[c][k]);
        float z = m * ws;
        if (GENERAL) {
          accB[c][k] += base;
          if (a.bias) z = fmaf(b[k], s[k], z);
        }
        dg[k] = dX[c][k] * z * slope;
        accG[c][k] += dg[k];
        const float dm = base * ws;
        v[0] = fmaf(dm, m, v[0]);
        v[1] += dm;
        y[c][k] = m;
        dX[c][k] = dm;
      }
      if (has_g && !shared_gate) store8<ALIGNED>((TY*)a.dg + row * a.lddg, dg, c, t, G, d);
    }
    if (a.post != BETTY_NORM_NONE) row_sums<2>(v, red, half, G, t);
    const float pm = a.post != BETTY_NORM_NONE ? v[0] * a.inv_d : 0.f, mean_dm = post_layer ? v[1] * a.inv_d : 0.f;
    TY* dy = (TY*)a.dy + row * a.lddy;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float o[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] = q * (dX[c][k] - y[c][k] * pm - mean_dm);
      store8<ALIGNED>(dy, o, c, t, G, d);
    }
    if (shared_gate) {
      const unsigned gate = (unsigned)row / a.per_gate;
      const int64_t g0 = (int64_t)gate * a.per_gate;
      const int64_t g1 = g0 + a.per_gate < a.rows ? g0 + a.per_gate : a.rows;
      if (row + 1 == g1 || row + 1 == last) {
        const bool whole = g0 >= first && g1 <= last;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          if (whole) store8<ALIGNED>((TY*)a.dg + gate * a.lddg, accG[c], c, t, G, d);
          else store8<ALIGNED>(a.gate_partials + (walker + gate) * d, accG[c], c, t, G, d);
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
      store8<ALIGNED>(out, accC[c], c, t, G, d);
      store8<ALIGNED>(out + d, accA[c], c, t, G, d);
      if (GENERAL && a.bias) {
        store8<ALIGNED>(out + 2 * (int64_t)d, accD[c], c, t, G, d);
        store8<ALIGNED>(out + 3 * (int64_t)d, accB[c], c, t, G, d);
      }
    }
  } else if (CH == 1) {                       // d <= 256: the block's warps are added in order through shared memory
    const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    for (int qn = 0; qn < nq; ++qn) {
      __syncthreads();
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float v = qn == 0 ? accC[0][k] : accA[0][k];
        if (GENERAL && qn >= 2) v = qn == 2 ? accD[0][k] : accB[0][k];
        combine[warp * 256 + column<ALIGNED>(0, k, t, 32)] = v;
      }
      __syncthreads();
      for (int j = threadIdx.x; j < d; j += blockDim.x) {
        float s = 0.f;
        for (int w = 0; w < warps; ++w) s += combine[w * 256 + j];
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

int backward_blocks(int64_t rows, int G) {
  const int threads = G == 32 ? SMALL_THREADS : G, per_block = threads / G;
  const int64_t want = (rows + per_block - 1) / per_block, most = (int64_t)current_sm_count() * (MAX_G / threads);
  return (int)(want < 1 ? 1 : (want < most ? want : most));
}

template <typename TX, typename TY, bool ALIGNED, int CH, bool GENERAL>
static betty_status launch_backward(cudaStream_t stream, const Args& a, float* dparams) {
  const int threads = a.G == 32 ? SMALL_THREADS : a.G, blocks = a.walkers / (threads / a.G);
  const size_t smem = a.G == 32 ? (size_t)(threads / 32) * 256 * sizeof(float) : 0;
  launch_pdl(k_backward<TX, TY, ALIGNED, CH, GENERAL>, dim3(blocks), dim3(threads), smem, stream, a);
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
template <typename TX, typename TY, bool ALIGNED, bool GENERAL>
static betty_status backward_chunks(cudaStream_t stream, const Args& a, float* dparams) {
  switch (chunks_of(a.d, a.G)) {
    case 1: return launch_backward<TX, TY, ALIGNED, 1, GENERAL>(stream, a, dparams);
    case 2: return launch_backward<TX, TY, ALIGNED, 2, GENERAL>(stream, a, dparams);
    default: return launch_backward<TX, TY, ALIGNED, 4, GENERAL>(stream, a, dparams);
  }
}
template <typename TX, typename TY>
static betty_status backward_typed(cudaStream_t stream, const Args& a, bool aligned, float* dparams) {
  const bool general = a.bias || a.pre == BETTY_NORM_LAYER || a.post == BETTY_NORM_LAYER;
  if (aligned) return general ? backward_chunks<TX, TY, true, true>(stream, a, dparams) : backward_chunks<TX, TY, true, false>(stream, a, dparams);
  return general ? backward_chunks<TX, TY, false, true>(stream, a, dparams) : backward_chunks<TX, TY, false, false>(stream, a, dparams);
}
betty_status backward(cudaStream_t stream, Args& a, int xd, int yd, bool aligned, float* dparams) {
  if (xd == BETTY_F32 && yd == BETTY_F32) return backward_typed<float, float>(stream, a, aligned, dparams);
  if (xd == BETTY_F32 && yd == BETTY_BF16) return backward_typed<float, __nv_bfloat16>(stream, a, aligned, dparams);
  if (xd == BETTY_F32 && yd == BETTY_F16) return backward_typed<float, __half>(stream, a, aligned, dparams);
  if (xd == BETTY_BF16 && yd == BETTY_BF16) return backward_typed<__nv_bfloat16, __nv_bfloat16>(stream, a, aligned, dparams);
  return backward_typed<__half, __half>(stream, a, aligned, dparams);
}

}  // namespace blocknorm
}  // namespace betty
