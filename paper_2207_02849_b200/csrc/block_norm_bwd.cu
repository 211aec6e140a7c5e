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

// dm of one chunk, 8 fp32 values, kept in the thread's own slots of x' and du: where x' is fp32 each in its column's place,
// else values 0 .. 3 in the 16 bytes of x' and 4 .. 7 in those of du, or (granules of two) a granule's two values in its
// words of x' and of du.  Columns beyond d keep their zeros.
template <int GR, typename TX>
__device__ __forceinline__ int park_at(int at_u, int c, int k, int t, int G) {      // k: a multiple of 4 (GR = 8) or any
  if (GR == 8) return sizeof(TX) == 4 ? ((c * 2 + k / 4) * G + t) * 16 : (c * G + t) * 16 + (k / 4) * at_u;
  return sizeof(TX) == 4 ? ((c * 8 + k) * G + t) * 4 : ((c * 4 + k / 2) * G + t) * 4 + (k % 2) * at_u;
}
template <int GR, typename TX>
__device__ __forceinline__ void park(char* slot, int at_u, const float (&v)[8], int c, int t, int G, int d) {
  static_assert(GR == 8 || sizeof(TX) == 4 || GR == 2, "16-bit rows are fetched in granules of 8 or 2");
#pragma unroll
  for (int k = 0; k < 8; k += GR == 8 ? 4 : 1)
    if (column<GR>(c, k, t, G) < d) {
      char* at = slot + park_at<GR, TX>(at_u, c, k, t, G);
      if constexpr (GR == 8) *(float4*)at = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
      else *(float*)at = v[k];
    }
}
template <int GR, typename TX>
__device__ __forceinline__ void unpark(float (&v)[8], const char* slot, int at_u, int c, int t, int G) {
#pragma unroll
  for (int k = 0; k < 8; k += GR == 8 ? 4 : 1) {
    const char* at = slot + park_at<GR, TX>(at_u, c, k, t, G);
    if constexpr (GR == 8) {
      const float4 w = *(const float4*)at;
      v[k] = w.x; v[k + 1] = w.y; v[k + 2] = w.z; v[k + 3] = w.w;
    } else {
      v[k] = *(const float*)at;
    }
  }
}

// Each walker (thread group) takes a contiguous share of the rows, so that the column sums stay in its registers; it writes
// them once, and k_backward_sums adds the blocks' sums in order.  Per row: the norms' sums over the fetched values, then dX
// (and with it everything that hangs off dm), then dy.  dm waits for its row's sum in the slots of x' and du, which are read
// by then.  A gate shared by rows needs one sum H = sum dX m per gate: dg = a'(g) s w_post H and A gains a(g) H when the
// walker leaves the gate, so A waits in shared memory.
template <typename TX, typename TY, int GR, bool PIPE, int CH, bool GENERAL>
__global__ void __launch_bounds__(MAX_G, 1) k_backward(const Args a) {
  __shared__ float red[2 * RED_VALUES * 16];
  extern __shared__ __align__(16) char slots[];
  pdl_enter();
  const int G = a.G, d = a.d, t = threadIdx.x & (G - 1), sub = threadIdx.x / G, subs = blockDim.x / G;
  const int64_t walker = (int64_t)blockIdx.x * subs + sub;
  const int64_t first = share_start(walker, a.rows, a.walkers), last = share_start(walker + 1, a.rows, a.walkers);
  const bool has_y = a.y != nullptr, has_g = a.gate != BETTY_GATE_NONE, has_u = a.du != nullptr, has_o = a.dxo != nullptr;
  const bool pre_layer = GENERAL && a.pre == BETTY_NORM_LAYER && has_u, post_layer = GENERAL && a.post == BETTY_NORM_LAYER && has_y;
  const bool shared_gate = has_g && a.per_gate > 1, row_gate = has_g && !shared_gate;
  const float* w_pre = a.params;
  const float* w_post = a.params + d;
  const float* s_res = a.params + 2 * (int64_t)d;
  const float* b_post = a.params + 4 * (int64_t)d;
  const int bx = CH * 8 * G * (int)sizeof(TX), by = CH * 8 * G * (int)sizeof(TY);
  const int at_o = bx, at_y = 2 * bx, at_u = 2 * bx + by, at_g = 2 * bx + 2 * by;
  char* ring = slots + (size_t)sub * (a.ahead + 1) * a.slot_bytes;
  // [A (, B)][value][thread] of a walker whose gates are shared
  float* acc_s = (float*)(slots + (size_t)subs * (a.ahead + 1) * a.slot_bytes) + (size_t)sub * (GENERAL ? 2 : 1) * CH * 8 * G + t;
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
        if (row_gate) copy_row<GR, CH>(p + at_g, (const TY*)a.g + r * a.ldg, t, G, d);
      }
      copies_commit();
    }
  };
  // one chunk of a stream of the present row
  char* p = nullptr;
  int64_t row = first;
  auto get = [&](auto* base, int64_t ld, int at, int c, float (&v)[8]) {
    typedef typename std::remove_const<typename std::remove_pointer<decltype(base)>::type>::type T;
    if constexpr (PIPE) read_slot<GR, T>(v, p + at, c, t, G);
    else load8<GR, T>(v, base + row * ld, c, t, G, d);
  };
  int half = 0, slot = 0;
  if constexpr (PIPE) {
    for (int i = 0; i <= a.ahead && CH * 8 * G > d; ++i) {
      char* s = ring + i * a.slot_bytes;
      clear_beyond<GR, CH, TX>(s, t, G, d);
      clear_beyond<GR, CH, TX>(s + at_o, t, G, d);
      clear_beyond<GR, CH, TY>(s + at_y, t, G, d);
      clear_beyond<GR, CH, TY>(s + at_u, t, G, d);
      if (row_gate) clear_beyond<GR, CH, TY>(s + at_g, t, G, d);
    }
    for (int i = 0; i < a.ahead; ++i) fetch(first + i, i);
  }
  // w_pre and w_post * s stay in registers (CH <= 2) or are read again
  constexpr bool KEEP = CH <= 2;
  float kp[KEEP ? CH : 1][8], kws[KEEP ? CH : 1][8], mask[GENERAL ? CH : 1][8 / GR];
  auto params_of = [&](int c, float (&wp)[8], float (&ws)[8]) {
    float s[8];
    load_param8<GR>(wp, w_pre, c, t, G, d);
    load_param8<GR>(ws, w_post, c, t, G, d);
    load_param8<GR>(s, s_res, c, t, G, d);
#pragma unroll
    for (int k = 0; k < 8; ++k) ws[k] *= s[k];
  };
  float accC[CH][8], accA[CH][8], accD[GENERAL ? CH : 1][8], accB[GENERAL ? CH : 1][8];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if constexpr (KEEP) params_of(c, kp[c], kws[c]);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      accC[c][k] = 0.f; accA[c][k] = 0.f;
      if (GENERAL) { accD[c][k] = 0.f; accB[c][k] = 0.f; }
      if (shared_gate) {
        acc_s[(c * 8 + k) * G] = 0.f;
        if (GENERAL) acc_s[(CH * 8 + c * 8 + k) * G] = 0.f;
      }
    }
    if (GENERAL)
#pragma unroll
      for (int k = 0; k < 8; k += GR) mask[c][k / GR] = column<GR>(c, k, t, G) < d ? 1.f : 0.f;   // 0 beyond the row
  }
  const TX* xs = (const TX*)a.x;
  const TX* os = (const TX*)a.dxo;
  const TY* ys = (const TY*)a.y;
  const TY* us = (const TY*)a.du;
  int64_t gate = 0, gate_end = 0;          // of a shared gate: the present row's, and the row after its last
  if (shared_gate && first < last) {
    gate = (unsigned)first / a.per_gate;
    gate_end = (gate + 1) * a.per_gate;
  }
  for (; row < last; ++row) {
    if (PIPE) {
      fetch(row + a.ahead, slot == 0 ? a.ahead : slot - 1);
      copies_wait(a.ahead);
      p = ring + slot * a.slot_bytes;
      slot = slot == a.ahead ? 0 : slot + 1;
    }
    float mean_dn = 0.f, mx = 0.f, my = 0.f;
    if (pre_layer || post_layer) {
      float v[3] = {0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        if (pre_layer) {
          float x[8], du[8], w[8], ws[8];
          get(xs, a.ldx, 0, c, x);
          get(us, a.lddu, at_u, c, du);
          if constexpr (!KEEP) params_of(c, w, ws);
#pragma unroll
          for (int k = 0; k < 8; ++k) { v[0] += x[k]; v[2] = fmaf(du[k], KEEP ? kp[KEEP ? c : 0][k] : w[k], v[2]); }
        }
        if (post_layer) {
          float y[8];
          get(ys, a.ldy, at_y, c, y);
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
          float x[8], du[8], w[8], ws[8];
          get(xs, a.ldx, 0, c, x);
          get(us, a.lddu, at_u, c, du);
          if constexpr (!KEEP) params_of(c, w, ws);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            if (GENERAL) x[k] = fmaf(-mx, mask[c][k / GR], x[k]);
            v[0] = fmaf(x[k], x[k], v[0]);
            v[1] = fmaf(du[k] * (KEEP ? kp[KEEP ? c : 0][k] : w[k]), x[k], v[1]);
          }
        }
        if (has_y) {
          float y[8];
          get(ys, a.ldy, at_y, c, y);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            if (GENERAL) y[k] = fmaf(-my, mask[c][k / GR], y[k]);
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
    float v[2] = {0.f, 0.f};
    // dm of the row: in registers where a thread holds one chunk (or nothing is fetched ahead), else over x' and du
    constexpr bool PARK = PIPE && CH > 1;
    float dm[PARK ? 1 : CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float dX[8], w[8], ws[8];
      if constexpr (!KEEP) params_of(c, w, ws);
      if (has_o) get(os, a.lddxo, at_o, c, dX);
      else
#pragma unroll
        for (int k = 0; k < 8; ++k) dX[k] = 0.f;
      if (has_u) {
        float x[8], du[8];
        get(xs, a.ldx, 0, c, x);
        get(us, a.lddu, at_u, c, du);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float n = (GENERAL ? fmaf(-mx, mask[c][k / GR], x[k]) : x[k]) * r;
          accC[c][k] = fmaf(du[k], n, accC[c][k]);
          if (GENERAL) accD[c][k] += du[k];
          float dn = fmaf(-n, proj, du[k] * (KEEP ? kp[KEEP ? c : 0][k] : w[k]));
          if (GENERAL) dn -= mean_dn;
          dX[k] = fmaf(r, dn, dX[k]);
        }
      }
      store8<GR>((TX*)a.dx + row * a.lddx, dX, c, t, G, d);
      if (!has_y) continue;
      float y[8], g[8], base[8];
      get(ys, a.ldy, at_y, c, y);
      if (shared_gate) load8<GR, TY>(g, (const TY*)a.g + gate * a.ldg, c, t, G, d);
      else if (row_gate) get((const TY*)a.g, a.ldg, at_g, c, g);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        y[k] = (GENERAL ? fmaf(-my, mask[c][k / GR], y[k]) : y[k]) * q;      // m
        if constexpr (KEEP) ws[k] = kws[KEEP ? c : 0][k];
      }
      if (has_g) {
        float slope[8];
        if (a.gate == BETTY_GATE_SIGMOID) {
#pragma unroll
          for (int k = 0; k < 8; ++k) { g[k] = sigmoid_f(g[k]); slope[k] = g[k] * (1.f - g[k]); }
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) slope[k] = 1.f;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) base[k] = dX[k] * g[k];
        if (shared_gate) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            accA[c][k] = fmaf(dX[k], y[k], accA[c][k]);
            if (GENERAL) accB[c][k] += dX[k];
          }
        } else {
          float dg[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) dg[k] = y[k] * ws[k];
          if (GENERAL && a.bias) {
            float b[8], s[8];
            load_param8<GR>(b, b_post, c, t, G, d);
            load_param8<GR>(s, s_res, c, t, G, d);
#pragma unroll
            for (int k = 0; k < 8; ++k) dg[k] = fmaf(b[k], s[k], dg[k]);
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) dg[k] *= dX[k] * slope[k];
          store8<GR>((TY*)a.dg + row * a.lddg, dg, c, t, G, d);
        }
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) base[k] = dX[k];
      }
      if (!shared_gate)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          accA[c][k] = fmaf(base[k], y[k], accA[c][k]);
          if (GENERAL) accB[c][k] += base[k];
        }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        base[k] *= ws[k];                                                    // dm
        v[0] = fmaf(base[k], y[k], v[0]);
        if (GENERAL) v[1] += base[k];
      }
      if constexpr (PARK) {
        park<GR, TX>(p, at_u, base, c, t, G, d);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) dm[PARK ? 0 : c][k] = base[k];
      }
    }
    if (!has_y) continue;
    if (a.post != BETTY_NORM_NONE) {
      if (GENERAL) row_sums<2>(v, red, half, G, t);
      else {
        float one[1] = {v[0]};
        row_sums<1>(one, red, half, G, t);
        v[0] = one[0];
      }
    }
    const float pm = a.post != BETTY_NORM_NONE ? v[0] * a.inv_d : 0.f, mean_dm = post_layer ? v[1] * a.inv_d : 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float o[8], y[8];
      get(ys, a.ldy, at_y, c, y);
      if constexpr (PARK) unpark<GR, TX>(o, p, at_u, c, t, G);
      else
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = dm[PARK ? 0 : c][k];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float m = (GENERAL ? fmaf(-my, mask[c][k / GR], y[k]) : y[k]) * q;
        o[k] = fmaf(-m, pm, o[k]);
        if (GENERAL) o[k] -= mean_dm;
        o[k] *= q;
      }
      store8<GR>((TY*)a.dy + row * a.lddy, o, c, t, G, d);
    }
    if (shared_gate && (row + 1 == gate_end || row + 1 == last)) {           // the walker leaves the gate
      const int64_t g0 = gate * a.per_gate, g1 = gate_end < a.rows ? gate_end : a.rows;
      const bool whole = g0 >= first && g1 <= last;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float g[8], dg[8], w[8], ws[8];
        if constexpr (!KEEP) params_of(c, w, ws);
        load8<GR, TY>(g, (const TY*)a.g + gate * a.ldg, c, t, G, d);
#pragma unroll
        for (int k = 0; k < 8; ++k) dg[k] = accA[c][k] * (KEEP ? kws[KEEP ? c : 0][k] : ws[k]);
        if (GENERAL && a.bias) {
          float b[8], s[8];
          load_param8<GR>(b, b_post, c, t, G, d);
          load_param8<GR>(s, s_res, c, t, G, d);
#pragma unroll
          for (int k = 0; k < 8; ++k) dg[k] = fmaf(b[k] * s[k], accB[c][k], dg[k]);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (a.gate == BETTY_GATE_SIGMOID) {
            g[k] = sigmoid_f(g[k]);
            dg[k] *= g[k] * (1.f - g[k]);
          }
          acc_s[(c * 8 + k) * G] = fmaf(g[k], accA[c][k], acc_s[(c * 8 + k) * G]);
          accA[c][k] = 0.f;
          if (GENERAL) {
            acc_s[(CH * 8 + c * 8 + k) * G] = fmaf(g[k], accB[c][k], acc_s[(CH * 8 + c * 8 + k) * G]);
            accB[c][k] = 0.f;
          }
        }
        if (whole) store8<GR>((TY*)a.dg + gate * a.lddg, dg, c, t, G, d);
        else store8<GR>(a.gate_partials + (walker + gate) * d, dg, c, t, G, d);
      }
      ++gate;
      gate_end += a.per_gate;
    }
  }
  const int nq = a.bias ? 4 : 2;
  float* out = a.col_partials + (int64_t)blockIdx.x * nq * d;
  if (shared_gate)
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        accA[c][k] = acc_s[(c * 8 + k) * G];
        if (GENERAL) accB[c][k] = acc_s[(CH * 8 + c * 8 + k) * G];
      }
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
        for (int w = 0; w < subs; ++w) s += combine[w * W + j];
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
static inline bool is_general(int bias, int pre, int post) { return bias || pre == BETTY_NORM_LAYER || post == BETTY_NORM_LAYER; }
// chunks per thread of the wide kernel: the layer norms' and biases' sums leave registers for one
static constexpr int backward_chunks(bool general) { return general ? 1 : 2; }
Layout backward_layout(const betty_block_norm_cfg* c, int64_t rows, int xd, int yd, int granule) {
  const bool gated = c->gate != BETTY_GATE_NONE, general = is_general(c->bias, c->pre, c->post);
  const bool row_gate = gated && c->rows_per_gate == 1;             // a gate shared by rows stays in L1
  Needs n = {2, row_gate ? 3 : 2, backward_chunks(general), 1, gated && !row_gate ? (general ? 2 : 1) : 0};
  Layout l = layout_of(c->d, rows, xd, yd, granule, n);
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
  constexpr int CH = backward_chunks(GENERAL), GR = sizeof(TY) == 4 ? 1 : 2;
  if (!l.ahead)
    return l.granule == 8 ? launch_backward<TX, TY, 8, false, 4, GENERAL>(stream, a, l, dparams)
                          : launch_backward<TX, TY, 1, false, 4, GENERAL>(stream, a, l, dparams);
  if (l.granule == 8)
    return l.wide ? launch_backward<TX, TY, 8, true, CH, GENERAL>(stream, a, l, dparams) : launch_backward<TX, TY, 8, true, 1, GENERAL>(stream, a, l, dparams);
  return l.wide ? launch_backward<TX, TY, GR, true, CH, GENERAL>(stream, a, l, dparams) : launch_backward<TX, TY, GR, true, 1, GENERAL>(stream, a, l, dparams);
}
template <typename TX, typename TY>
static betty_status backward_typed(cudaStream_t stream, const Args& a, const Layout& l, float* dparams) {
  return is_general(a.bias, a.pre, a.post) ? backward_shape<TX, TY, true>(stream, a, l, dparams) : backward_shape<TX, TY, false>(stream, a, l, dparams);
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
