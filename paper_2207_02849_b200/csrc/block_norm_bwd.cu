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




// Each walker (thread group) takes a contiguous share of the rows, so that the column sums stay in its registers; it writes
// them once, and k_backward_sums adds the blocks' sums in order.  A row's chain is what bounds this kernel, so with RMS
// norms a row costs one sum over its threads: with c = a w_post s y the mean of dm m is a combination of sums that do not
// wait for dX,
//
//   <dm m> d = q (sum dx' c + r sum dn0 c - r^2 proj sum x' c),   dn0 = du w_pre,   proj = <dn n>
//
// and then dX, dm, dy and all products of the row come out in one go.  Layer norms take the means first and <dm>, <dm m>
// from dm itself: their combination would cancel two differences that are scaled up by 1 / sigma each where rows are flat.
// A gate shared by rows needs one sum H = sum dX m per gate: dg = a'(g) s w_post H, and A gains a(g) H when the walker
// leaves the gate, so A waits in shared memory.
template <typename TX, typename TY, int GR, bool PIPE, int CH, bool GENERAL>
__global__ void __launch_bounds__(MAX_G, 1) k_backward(const Args a) {
  __shared__ float red[2 * RED_VALUES * 16];
  extern __shared__ __align__(16) char slots[];      // fetched rows; G = 32: at the end the warps' column sums
  pdl_enter();
  const int G = a.G, d = a.d, t = threadIdx.x & (G - 1), sub = threadIdx.x / G, subs = blockDim.x / G;
  const int64_t walker = (int64_t)blockIdx.x * subs + sub;
  const int64_t first = walker < a.walkers ? share_start(walker, a.rows, a.walkers) : a.rows;
  const int64_t last = walker < a.walkers ? share_start(walker + 1, a.rows, a.walkers) : a.rows;
  const bool has_y = a.y != nullptr, has_g = a.gate != BETTY_GATE_NONE, has_u = a.du != nullptr, has_o = a.dxo != nullptr;
  const bool pre_layer = GENERAL && a.pre == BETTY_NORM_LAYER && has_u, post_layer = GENERAL && a.post == BETTY_NORM_LAYER && has_y;
  const bool shared_gate = has_g && a.per_gate > 1, row_gate = has_g && !shared_gate, bias = GENERAL && a.bias;
  const float* w_pre = a.params;
  const float* w_post = a.params + d;
  const float* s_res = a.params + 2 * (int64_t)d;
  const float* b_post = a.params + 4 * (int64_t)d;
  const int bx = CH * 8 * G * (int)sizeof(TX), by = CH * 8 * G * (int)sizeof(TY);
  const int at_o = bx, at_y = 2 * bx, at_u = 2 * bx + by, at_g = 2 * bx + 2 * by;
  char* ring = slots + (size_t)sub * (a.ahead + 1) * a.slot_bytes;
  // [A (, B)][value][thread] of a walker whose gates are shared
  // w_pre of the block, then e of each walker: [half chunk][thread], read with 16-byte accesses
  float4* w_s = (float4*)(slots + (size_t)subs * (a.ahead + 1) * a.slot_bytes) + t;
  float4* e_s = w_s + (size_t)(sub + 1) * 2 * CH * G;
  // A (and B) of a walker whose gates are shared: its block's row of the column sums, or where a warp holds a row (several
  // walkers to a block) [value][thread] in shared memory
  float* acc_s = (float*)(w_s - t + (size_t)(subs + 1) * 2 * CH * G) + (size_t)sub * (GENERAL ? 2 : 1) * CH * 8 * G + t;
  float* const partials = a.col_partials + (int64_t)blockIdx.x * (a.bias ? 4 : 2) * d;
  const TX* xs = (const TX*)a.x;
  const TX* os = (const TX*)a.dxo;
  const TY* ys = (const TY*)a.y;
  const TY* us = (const TY*)a.du;
  const TY* gs = (const TY*)a.g;
  auto fetch = [&](int64_t r, int slot) {
    if constexpr (PIPE) {
      if (r < last) {
        char* p = ring + slot * a.slot_bytes;
        if (has_u) {
          copy_row<GR, CH>(p, xs + r * a.ldx, t, G, d);
          copy_row<GR, CH>(p + at_u, us + r * a.lddu, t, G, d);
        }
        if (has_o) copy_row<GR, CH>(p + at_o, os + r * a.lddxo, t, G, d);
        if (has_y) copy_row<GR, CH>(p + at_y, ys + r * a.ldy, t, G, d);
        if (row_gate) copy_row<GR, CH>(p + at_g, gs + r * a.ldg, t, G, d);
      }
      copies_commit();
    }
  };
  // one chunk of a stream of the present row
  const char* p = nullptr;
  int64_t row = first;
  auto get = [&](auto* base, int64_t ld, int at, int c, f2 (&o)[4]) {
    typedef typename std::remove_const<typename std::remove_pointer<decltype(base)>::type>::type T;
    float v[8];
    if constexpr (PIPE) read_slot<GR, T>(v, p + at, c, t, G);
    else load8<GR, T>(v, base + row * ld, c, t, G, d);
    pairs(o, v);
  };
  auto param = [&](const float* base, int c, f2 (&o)[4]) {
    float v[8];
    load_param8<GR>(v, base, c, t, G, d);
    pairs(o, v);
  };
  int half = 0, slot = 0;
  if (PIPE)
    for (int i = 0; i < a.ahead; ++i) fetch(first + i, i);

  int64_t gate = 0, gate_end = 0;          // of a shared gate: the present row's, and the row after its last
  if (shared_gate && first < last) {
    gate = (unsigned)first / a.per_gate;
    gate_end = (gate + 1) * a.per_gate;
  }
  // w_pre and e = w_post s, times a(g) of a shared gate: in shared memory; wide rows form them where they are used
  constexpr bool KEEP = CH <= 2;
  auto make_e = [&](int c, f2 (&e)[4]) {
    f2 s[4];
    param(w_post, c, e);
    param(s_res, c, s);
#pragma unroll
    for (int k = 0; k < 4; ++k) e[k] = mul2(e[k], s[k]);
    if (shared_gate) {
      float g[8];
      load8<GR, TY>(g, gs + gate * a.ldg, c, t, G, d);
      if (a.gate == BETTY_GATE_SIGMOID)
#pragma unroll
        for (int k = 0; k < 8; ++k) g[k] = sigmoid_f(g[k]);
      pairs(s, g);
#pragma unroll
      for (int k = 0; k < 4; ++k) e[k] = mul2(e[k], s[k]);
    }
  };
  auto keep_e = [&](int c) {
    f2 e[4];
    make_e(c, e);
    e_s[(2 * c) * G] = make_float4(e[0].x, e[0].y, e[1].x, e[1].y);
    e_s[(2 * c + 1) * G] = make_float4(e[2].x, e[2].y, e[3].x, e[3].y);
  };
  auto coefficients = [&](int c, f2 (&w)[4], f2 (&e)[4]) {
    if constexpr (KEEP) {
      const float4 a0 = w_s[(2 * c) * G], a1 = w_s[(2 * c + 1) * G], b0 = e_s[(2 * c) * G], b1 = e_s[(2 * c + 1) * G];
      w[0] = f2{a0.x, a0.y}; w[1] = f2{a0.z, a0.w}; w[2] = f2{a1.x, a1.y}; w[3] = f2{a1.z, a1.w};
      e[0] = f2{b0.x, b0.y}; e[1] = f2{b0.z, b0.w}; e[2] = f2{b1.x, b1.y}; e[3] = f2{b1.z, b1.w};
    } else {
      param(w_pre, c, w);
      make_e(c, e);
    }
  };
  f2 accC[CH][4], accA[CH][4], accD[GENERAL ? CH : 1][4], accB[GENERAL ? CH : 1][4], mask[GENERAL ? CH : 1][4];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if constexpr (KEEP) {
      float w[8];
      load_param8<GR>(w, w_pre, c, t, G, d);         // every thread group writes the same values, and reads its own writes
      w_s[(2 * c) * G] = make_float4(w[0], w[1], w[2], w[3]);
      w_s[(2 * c + 1) * G] = make_float4(w[4], w[5], w[6], w[7]);
      keep_e(c);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      accC[c][k] = accA[c][k] = both(0.f);
      if (GENERAL) {
        accD[c][k] = accB[c][k] = both(0.f);
        mask[c][k] = f2{column<GR>(c, 2 * k, t, G) < d ? 1.f : 0.f, column<GR>(c, 2 * k + 1, t, G) < d ? 1.f : 0.f};   // 0 beyond the row
      }
    }
    if (shared_gate) {
      float zero[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        zero[k] = 0.f;
        if (G == 32) {
          acc_s[(c * 8 + k) * G] = 0.f;
          if (GENERAL) acc_s[(CH * 8 + c * 8 + k) * G] = 0.f;
        }
      }
      if (G > 32) {
        store8<GR>(partials + d, zero, c, t, G, d);
        if (bias) store8<GR>(partials + 3 * (int64_t)d, zero, c, t, G, d);
      }
    }
  }
  for (; row < last; ++row) {
    if (PIPE) {
      fetch(row + a.ahead, slot == 0 ? a.ahead : slot - 1);
      copies_wait(a.ahead);
      p = ring + slot * a.slot_bytes;
      slot = slot == a.ahead ? 0 : slot + 1;
    }
    float mx = 0.f, my = 0.f;
    if (pre_layer || post_layer) {
      f2 sx = both(0.f), sy = both(0.f);
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        f2 v[4];
        if (pre_layer) {
          get(xs, a.ldx, 0, c, v);
#pragma unroll
          for (int k = 0; k < 4; ++k) sx = add2(sx, v[k]);
        }
        if (post_layer) {
          get(ys, a.ldy, at_y, c, v);
#pragma unroll
          for (int k = 0; k < 4; ++k) sy = add2(sy, v[k]);
        }
      }
      float v[2] = {sx.x + sx.y, sy.x + sy.y};
      row_sums<2>(v, red, half, G, t);
      if (pre_layer) mx = v[0] * a.inv_d;
      if (post_layer) my = v[1] * a.inv_d;
    }
    // x2, dn0 x, y2, and dx' c, dn0 c, x c; layer norms dn0
    constexpr int NS = GENERAL ? 4 : 6;
    float S[NS];
    {
      f2 s2[NS];
#pragma unroll
      for (int i = 0; i < NS; ++i) s2[i] = both(0.f);
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        f2 x[4], u[4], w[4], e[4];
        coefficients(c, w, e);
        if (has_u) {
          get(xs, a.ldx, 0, c, x);
          get(us, a.lddu, at_u, c, u);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (GENERAL) x[k] = fma2(both(-mx), mask[c][k], x[k]);
            u[k] = mul2(u[k], w[k]);
            s2[0] = fma2(x[k], x[k], s2[0]);
            s2[1] = fma2(u[k], x[k], s2[1]);
            if (GENERAL) s2[3] = add2(s2[3], u[k]);
          }
        }
        if (has_y) {
          f2 y[4];
          get(ys, a.ldy, at_y, c, y);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (GENERAL) y[k] = fma2(both(-my), mask[c][k], y[k]);
            s2[2] = fma2(y[k], y[k], s2[2]);
          }
          if constexpr (!GENERAL) {
            if (row_gate) {
              f2 g[4];
              get(gs, a.ldg, at_g, c, g);
              if (a.gate == BETTY_GATE_SIGMOID)
#pragma unroll
                for (int k = 0; k < 4; ++k) g[k] = f2{sigmoid_f(g[k].x), sigmoid_f(g[k].y)};
#pragma unroll
              for (int k = 0; k < 4; ++k) e[k] = mul2(e[k], g[k]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = mul2(y[k], e[k]);               // c
            if (has_u)
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                s2[4] = fma2(u[k], y[k], s2[4]);
                s2[5] = fma2(x[k], y[k], s2[5]);
              }
            if (has_o) {
              f2 o[4];
              get(os, a.lddxo, at_o, c, o);
#pragma unroll
              for (int k = 0; k < 4; ++k) s2[3] = fma2(o[k], y[k], s2[3]);
            }
          }
        }
      }
#pragma unroll
      for (int i = 0; i < NS; ++i) S[i] = s2[i].x + s2[i].y;
      row_sums<NS>(S, red, half, G, t);
    }
    float r = 1.f, q = 1.f, cx = 0.f, mean_dn = 0.f;      // dX = dx' + r (dn0 - <dn>) + cx (x - mean)
    if (a.pre != BETTY_NORM_NONE && has_u) {
      r = rsqrtf(fmaf(S[0], a.inv_d, a.eps));
      cx = -r * r * r * S[1] * a.inv_d;
      if (pre_layer) mean_dn = S[3] * a.inv_d;
    }
    float pm = 0.f;
    if (a.post != BETTY_NORM_NONE && has_y) {
      q = rsqrtf(fmaf(S[2], a.inv_d, a.eps));
      if constexpr (!GENERAL) pm = q * fmaf(r, S[NS - 2], fmaf(cx, S[NS - 1], S[3])) * a.inv_d;
    }
    const f2 r2 = both(r), cx2 = both(cx), q2 = both(q), pq2 = both(-pm * q), dn2 = both(-mean_dn);
    f2 dm[GENERAL ? CH : 1][4], sm = both(0.f), sd = both(0.f);       // layer norms: dm, sum dm m, sum dm
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      f2 dX[4], w[4], e[4];
      float out[8];
      coefficients(c, w, e);
      if (has_o) get(os, a.lddxo, at_o, c, dX);
      else
#pragma unroll
        for (int k = 0; k < 4; ++k) dX[k] = both(0.f);
      if (has_u) {
        f2 x[4], u[4];
        get(xs, a.ldx, 0, c, x);
        get(us, a.lddu, at_u, c, u);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (GENERAL) x[k] = fma2(both(-mx), mask[c][k], x[k]);
          dX[k] = fma2(x[k], cx2, dX[k]);
          f2 dn = mul2(u[k], w[k]);
          if (GENERAL) dn = add2(dn, dn2);          // subtracted before the scaling: r can be large where a row is flat
          dX[k] = fma2(dn, r2, dX[k]);
          if (GENERAL) {
            accD[c][k] = add2(accD[c][k], u[k]);
          }
          accC[c][k] = fma2(u[k], mul2(x[k], r2), accC[c][k]);
        }
      }
      singles(out, dX);
      store8<GR>((TX*)a.dx + row * a.lddx, out, c, t, G, d);
      if (!has_y) continue;
      f2 m[4];
      get(ys, a.ldy, at_y, c, m);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (GENERAL) m[k] = fma2(both(-my), mask[c][k], m[k]);
        m[k] = mul2(m[k], q2);
      }
      if (row_gate) {
        f2 g[4], z[4];
        get(gs, a.ldg, at_g, c, g);
#pragma unroll
        for (int k = 0; k < 4; ++k) z[k] = mul2(m[k], e[k]);
        if (bias) {
          f2 b[4], s[4];
          param(b_post, c, b);
          param(s_res, c, s);
#pragma unroll
          for (int k = 0; k < 4; ++k) z[k] = fma2(b[k], s[k], z[k]);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) z[k] = mul2(z[k], dX[k]);
        if (a.gate == BETTY_GATE_SIGMOID)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            g[k] = f2{sigmoid_f(g[k].x), sigmoid_f(g[k].y)};
            z[k] = mul2(z[k], fma2(mul2(g[k], both(-1.f)), g[k], g[k]));
          }
        singles(out, z);
        store8<GR>((TY*)a.dg + row * a.lddg, out, c, t, G, d);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          dX[k] = mul2(dX[k], g[k]);
          if (GENERAL) accB[c][k] = add2(accB[c][k], dX[k]);
        }
      } else if (GENERAL) {
#pragma unroll
        for (int k = 0; k < 4; ++k) accB[c][k] = add2(accB[c][k], dX[k]);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        accA[c][k] = fma2(dX[k], m[k], accA[c][k]);
        dX[k] = mul2(dX[k], e[k]);                                 // dm
        if constexpr (GENERAL) {
          dm[c][k] = dX[k];
          sm = fma2(dX[k], m[k], sm);
          sd = add2(sd, dX[k]);
        } else {
          const f2 o = fma2(dX[k], q2, mul2(m[k], pq2));           // q (dm - m <dm m>)
          out[2 * k] = o.x; out[2 * k + 1] = o.y;
        }
      }
      if (!GENERAL) store8<GR>((TY*)a.dy + row * a.lddy, out, c, t, G, d);
    }
    if constexpr (GENERAL) {
      if (has_y) {
        float v[2] = {sm.x + sm.y, sd.x + sd.y};
        if (a.post != BETTY_NORM_NONE) row_sums<2>(v, red, half, G, t);
        const float mean = post_layer ? v[1] * a.inv_d : 0.f;
        pm = a.post != BETTY_NORM_NONE ? v[0] * a.inv_d : 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          f2 m[4];
          float out[8];
          get(ys, a.ldy, at_y, c, m);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            m[k] = mul2(fma2(both(-my), mask[c][k], m[k]), q2);
            const f2 o = mul2(fma2(m[k], both(-pm), add2(dm[c][k], both(-mean))), q2);      // q (dm - <dm> - m <dm m>)
            out[2 * k] = o.x; out[2 * k + 1] = o.y;
          }
          store8<GR>((TY*)a.dy + row * a.lddy, out, c, t, G, d);
        }
      }
    }
    if (has_y && shared_gate && (row + 1 == gate_end || row + 1 == last)) {           // the walker leaves the gate
      const int64_t g0 = gate * a.per_gate, g1 = gate_end < a.rows ? gate_end : a.rows;
      const bool whole = g0 >= first && g1 <= last;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float g[8], dg[8], w[8], s[8], b[8];
        load8<GR, TY>(g, gs + gate * a.ldg, c, t, G, d);
        load_param8<GR>(w, w_post, c, t, G, d);
        load_param8<GR>(s, s_res, c, t, G, d);
        if (bias) load_param8<GR>(b, b_post, c, t, G, d);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float H = k & 1 ? accA[c][k / 2].y : accA[c][k / 2].x, E = !GENERAL ? 0.f : (k & 1 ? accB[GENERAL ? c : 0][k / 2].y : accB[GENERAL ? c : 0][k / 2].x);
          dg[k] = s[k] * (bias ? fmaf(b[k], E, w[k] * H) : w[k] * H);
          if (a.gate == BETTY_GATE_SIGMOID) {
            g[k] = sigmoid_f(g[k]);
            dg[k] *= g[k] * (1.f - g[k]);
          }
          if (G == 32) {
            acc_s[(c * 8 + k) * G] = fmaf(g[k], H, acc_s[(c * 8 + k) * G]);
            if (GENERAL) acc_s[(CH * 8 + c * 8 + k) * G] = fmaf(g[k], E, acc_s[(CH * 8 + c * 8 + k) * G]);
          } else {
            w[k] = g[k] * H;
            if (GENERAL) b[k] = g[k] * E;
          }
        }
        if (G > 32) {
          float was[8];
          load8<GR, float>(was, partials + d, c, t, G, d);
#pragma unroll
          for (int k = 0; k < 8; ++k) w[k] += was[k];
          store8<GR>(partials + d, w, c, t, G, d);
          if (bias) {
            load8<GR, float>(was, partials + 3 * (int64_t)d, c, t, G, d);
#pragma unroll
            for (int k = 0; k < 8; ++k) b[k] += was[k];
            store8<GR>(partials + 3 * (int64_t)d, b, c, t, G, d);
          }
        }
        if (whole) store8<GR>((TY*)a.dg + gate * a.lddg, dg, c, t, G, d);
        else store8<GR>(a.gate_partials + (walker + gate) * d, dg, c, t, G, d);
      }
      ++gate;
      gate_end += a.per_gate;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          accA[c][k] = both(0.f);
          if (GENERAL) accB[c][k] = both(0.f);
        }
        if constexpr (KEEP)
          if (row + 1 < last) keep_e(c);
      }
    }
  }
  if (shared_gate && G == 32)
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        accA[c][k] = f2{acc_s[(c * 8 + 2 * k) * G], acc_s[(c * 8 + 2 * k + 1) * G]};
        if (GENERAL) accB[c][k] = f2{acc_s[(CH * 8 + c * 8 + 2 * k) * G], acc_s[(CH * 8 + c * 8 + 2 * k + 1) * G]};
      }
  const int nq = a.bias ? 4 : 2;
  float* out = partials;
  float* combine = (float*)slots;             // G = 32, a warp per walker: the block's warps are added in order
  constexpr int W = CH * 256;                 // columns a warp can hold
  for (int qn = 0; qn < nq; ++qn, out += d) {
    if (shared_gate && G > 32 && (qn & 1)) continue;       // A and B are there already
    if (G == 32) __syncthreads();
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float v[8];
      if (qn == 0) singles(v, accC[c]);
      else if (!GENERAL || qn == 1) singles(v, accA[c]);
      else singles(v, qn == 2 ? accD[GENERAL ? c : 0] : accB[GENERAL ? c : 0]);
      if (G > 32) store8<GR>(out, v, c, t, G, d);
      else
#pragma unroll
        for (int k = 0; k < 8; ++k) combine[sub * W + column<GR>(c, k, t, 32)] = v[k];
    }
    if (G == 32) {
      __syncthreads();
      for (int j = threadIdx.x; j < d; j += blockDim.x) {
        float s = 0.f;
        for (int w = 0; w < subs; ++w) s += combine[w * W + j];
        out[j] = s;
      }
    }
  }
}

// Adds the blocks' column sums and forms the parameter gradients (the first param_blocks blocks: 32 columns each, SLICES
// slices of the list added in a fixed order), then the gates whose rows lie in several walkers' shares.
static constexpr int SLICES = 16, GATE_COLUMNS = 128;
template <typename TY>
__global__ void __launch_bounds__(32 * SLICES) k_backward_sums(const Args a, int blocks, int param_blocks, float* __restrict__ dparams) {
  __shared__ float part[4][SLICES][32];
  pdl_enter();
  const int d = a.d;
  if ((int)blockIdx.x < param_blocks) {
    const int j = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5, nq = a.bias ? 4 : 2;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (j < d) {
      const float* p = a.col_partials + (int64_t)slice * nq * d + j;
      const int64_t step = (int64_t)SLICES * nq * d;
      if (nq == 2) {
#pragma unroll 10
        for (int b = slice; b < blocks; b += SLICES, p += step) { v[0] += p[0]; v[1] += p[d]; }
      } else {
#pragma unroll 5
        for (int b = slice; b < blocks; b += SLICES, p += step) { v[0] += p[0]; v[1] += p[d]; v[2] += p[2 * (int64_t)d]; v[3] += p[3 * (int64_t)d]; }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) part[i][slice][threadIdx.x & 31] = v[i];
    __syncthreads();
    if (slice == 0 && j < d) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = 0.f;
#pragma unroll
        for (int s = 0; s < SLICES; ++s) v[i] += part[i][s][threadIdx.x];
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
  const int col_blocks = (d + GATE_COLUMNS - 1) / GATE_COLUMNS;
  const int item = (blockIdx.x - param_blocks) / col_blocks, lane = threadIdx.x % GATE_COLUMNS, slice = threadIdx.x / GATE_COLUMNS;
  const int j = ((blockIdx.x - param_blocks) % col_blocks) * GATE_COLUMNS + lane;
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
  if (lo == hi) return;
  // the walkers in between, in slices added in a fixed order; there are no more walkers than rows, so none is empty
  constexpr int GS = 32 * SLICES / GATE_COLUMNS;
  float s = 0.f;
  if (j < d) {
    const float* p = a.gate_partials + (lo + slice + gate) * d + j;
#pragma unroll 8
    for (int64_t w = lo + slice; w <= hi; w += GS, p += (int64_t)GS * d) s += *p;
  }
  float* sums = &part[0][0][0];
  sums[slice * GATE_COLUMNS + lane] = s;
  __syncthreads();
  if (slice == 0 && j < d) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < GS; ++i) s += sums[i * GATE_COLUMNS + lane];
    ((TY*)a.dg)[gate * a.lddg + j] = from_f<TY>(s);
  }
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
  Needs n = {2, row_gate ? 3 : 2, backward_chunks(general), 1, 0, 1};
  n.acc_arrays = gated && !row_gate && c->d <= 32 * 8 * MAX_CH ? 1 + (general ? 2 : 1) : 1;      // e; A (and B) where a warp holds a row
  Layout l = layout_of(c->d, rows, xd, yd, granule, n);
  const size_t combine = l.G == 32 ? (size_t)(l.threads / 32) * l.chunks * 256 * sizeof(float) : 0;
  if (l.smem < combine) l.smem = combine;
  return l;
}

template <typename TX, typename TY, int GR, bool PIPE, int CH, bool GENERAL>
static betty_status launch_backward(cudaStream_t stream, const Args& a, const Layout& l, float* dparams) {
  static SmemLimit limit = {};
  if (l.smem > 40 * 1024) BETTY_TRY(ensure_dynamic_smem(k_backward<TX, TY, GR, PIPE, CH, GENERAL>, limit, l.smem));
  const int blocks = backward_blocks(a.rows, l);
  launch_pdl(k_backward<TX, TY, GR, PIPE, CH, GENERAL>, dim3(blocks), dim3(l.threads), l.smem, stream, a);
  BETTY_LAUNCH_CHECK();
  const int param_blocks = (a.d + 31) / 32;
  int64_t items = 0;
  if (a.gate_partials && a.rows > 0) {
    const int64_t gates = (a.rows + a.per_gate - 1) / a.per_gate;
    items = gates < a.walkers ? gates : a.walkers - 1;
  }
  launch_pdl(k_backward_sums<TY>, dim3((unsigned)(param_blocks + items * ((a.d + GATE_COLUMNS - 1) / GATE_COLUMNS))), dim3(32 * SLICES), 0, stream, a,
             blocks, param_blocks,
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
