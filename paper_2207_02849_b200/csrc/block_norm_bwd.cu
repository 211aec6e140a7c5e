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

// The rows of a class (row numbers equal modulo `classes`) are cut into `shares` contiguous shares, equal to within a row.
__device__ __forceinline__ int64_t class_rows(const Args& a, int kind) { return a.rows > kind ? (a.rows - kind + a.classes - 1) / a.classes : 0; }
__device__ __forceinline__ int64_t share_start(int64_t share, int64_t n, int shares) { return share * n / shares; }
__device__ __forceinline__ int64_t share_of(int64_t i, int64_t n, int shares) { return ((i + 1) * shares - 1) / n; }

// a row of sums in the workspace: 16 bytes at a time where that fits
template <bool VEC>
__device__ __forceinline__ void store_sums(float* row, const float (&v)[8], int c, const Place& w) {
  if (VEC && w.shift == 0 && w.d % 4 == 0) store8<VEC>(row, v, c, w);
  else store_each<VEC>(row, v, c, w);
}
// Where a walker's sum for a gate of several rows waits to be added to the other walkers'.  One class: a share has at most two
// gates that are not all its own, one that began before it and one that `begins` in it and goes on behind it.  Several
// classes: shares and gates both grow along the rows, so no two pairs of a class meet at share + gate; where that is more
// places than the class has rows (gates of few rows), a pair's place is its last row.
__device__ __forceinline__ unsigned first_slot(const Args& a, int kind, unsigned share) {
  return (unsigned)kind * (unsigned)a.gate_sums.rows + a.gate_sums.per_share * share;
}
__device__ __forceinline__ unsigned gate_slot(const Args& a, unsigned first, unsigned gate, bool begins, unsigned last_row) {
  return first + a.gate_sums.per_gate * gate + a.gate_sums.per_row * last_row + (begins ? a.gate_sums.begins : 0u);
}

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
// leaves the gate, so A waits in the block's row of the column sums.
//
// Measured: 8192 x 4096 bf16, RMS norms, gates of 1024 rows: 99 us (4.1 TB/s) against 62 us for the bytes; 2731 x 1537 fp32, layer
// norms with biases: 68 us against 21.  Neither pipe is full: the first issues 53 % of the time and uses 48 % of the memory, the
// second 34 and 18 %, with 16 warps per SM (two blocks of 256 threads at 128 registers): what is exposed is a row's own chain,
// from its values over two walks with the sums and a barrier between them.  SHARED (gates of several rows) is a template parameter
// because what such a gate needs took registers from every row: 130 -> 105 us with one, 115 -> 93 without any gate (single launches,
// cold).  Before that, two chunks per thread with the coefficients in shared memory took 123 us where registers for them spilled and
// took 153; one chunk per thread and 512 threads per row 141; two rows at a time 178 to 201 (spills).
template <typename TX, typename TY, bool VEC, int CH, bool GENERAL, bool SHARED>
__global__ void __launch_bounds__(MAX_G, 1) k_backward(const Args a) {
  __shared__ __align__(16) float red[2 * RED_VALUES * 16];
  extern __shared__ __align__(16) char slots[];      // fetched rows; G = 32: at the end the warps' column sums
  row_sums_init(red);
  pdl_enter();
  const int G = a.G, d = a.d, t = G == 32 ? threadIdx.x & 31 : threadIdx.x, sub = G == 32 ? threadIdx.x >> 5 : 0, subs = G == 32 ? blockDim.x >> 5 : 1;
  // walker: share `share` of the rows kind, kind + classes, ...; `at` and `last` count those
  const int walker = blockIdx.x * subs + sub, kind = walker % a.classes, share = walker / a.classes;
  const int64_t n_rows = class_rows(a, kind);
  // (row numbers and what is added to them stay below 2^32: a call has at most 2^31 - 1 rows, and so has a gate)
  const unsigned first = share < a.shares ? (unsigned)share_start(share, n_rows, a.shares) : (unsigned)n_rows;
  const unsigned last = share < a.shares ? (unsigned)share_start(share + 1, n_rows, a.shares) : (unsigned)n_rows;
  const Place pl = {t, G, d, VEC ? (int)((kind * a.ld8) & 7) : 0};
  auto row_of = [&](unsigned i) { return (unsigned)kind + i * (unsigned)a.classes; };
  const bool has_y = a.y != nullptr, has_g = a.gate != BETTY_GATE_NONE, has_u = a.du != nullptr, has_o = a.dxo != nullptr;
  const bool pre_layer = GENERAL && a.pre == BETTY_NORM_LAYER && has_u, post_layer = GENERAL && a.post == BETTY_NORM_LAYER && has_y;
  const bool shared_gate = SHARED, row_gate = has_g && !SHARED, bias = GENERAL && a.bias;
  const float* w_pre = a.params;
  const float* w_post = a.params + d;
  const float* s_res = a.params + 2 * (int64_t)d;
  const float* b_post = a.params + 4 * (int64_t)d;
  const int bx = CH * 8 * G * (int)sizeof(TX), by = CH * 8 * G * (int)sizeof(TY);
  const int at_o = bx, at_y = 2 * bx, at_u = 2 * bx + by, at_g = 2 * bx + 2 * by;
  // shared memory: the walkers' slots; then for each walker w_pre, e (and b_post s) of its columns, [half chunk][thread]; then A (and B)
  // of walkers whose gates are shared, where a warp holds a row (several walkers to a block), [value][thread] (elsewhere A
  // and B wait in the block's row of the column sums)
  const uint32_t base_s = shared_address(slots), slots_end = base_s + subs * (a.ahead + 1) * a.slot_bytes;
  const uint32_t ring = base_s + sub * (a.ahead + 1) * a.slot_bytes;
  constexpr int KEPT = GENERAL ? 6 : 4;      // half chunks of w_pre, e (and b_post s) for each chunk
  const uint32_t w_s = slots_end + (sub * KEPT * CH * G + t) * 16, e_s = w_s + 2 * CH * G * 16, b_s = e_s + 2 * CH * G * 16;
  constexpr bool KEEP = CH <= 2;             // wide rows form w_pre and e where they are used
  const uint32_t acc_s = slots_end + (KEEP ? subs * KEPT * CH * G * 16 : 0) + (sub * (GENERAL ? 2 : 1) * CH * 8 * G + t) * 4;
  float* const partials = a.col_partials + (int64_t)blockIdx.x * (a.bias ? 4 : 2) * d;
  const TX* const xs = (const TX*)a.x;
  const TX* const os = (const TX*)a.dxo;
  const TY* const ys = (const TY*)a.y;
  const TY* const us = (const TY*)a.du;
  const TY* const gs = (const TY*)a.g;
  auto fetch = [&](unsigned i, int slot) {
    if constexpr (VEC) {
      if (i < last) {
        const unsigned r = row_of(i);
        const uint32_t p = ring + slot * a.slot_bytes;
        if (has_u) {
          copy_row<CH>(p, row_at<TX>(xs, r, a.ldx), pl);
          copy_row<CH>(p + at_u, row_at<TY>(us, r, a.lddu), pl);
        }
        if (has_o) copy_row<CH>(p + at_o, row_at<TX>(os, r, a.lddxo), pl);
        if (has_y) copy_row<CH>(p + at_y, row_at<TY>(ys, r, a.ldy), pl);
        if (row_gate) copy_row<CH>(p + at_g, row_at<TY>(gs, r, a.ldg), pl);
      }
      copies_commit();
      if (CH == 2 && a.ahead == 0) copies_commit();      // an empty group behind the present row's: copies_wait leaves one in flight
    }
  };
  // one chunk of a stream of the present row
  uint32_t p = 0;
  unsigned row = 0;
  auto get = [&](auto* base, uint32_t ld, int at, int c, f2 (&o)[4]) {
    typedef typename std::remove_const<typename std::remove_pointer<decltype(base)>::type>::type T;
    float v[8];
    if constexpr (VEC) read_slot<T>(v, p + at, c, pl);
    else load8<VEC, T>(v, row_at<T>(base, row, ld), c, pl);
    pairs(o, v);
  };
  auto param = [&](const float* base, int c, f2 (&o)[4]) {
    float v[8];
    load8<VEC>(v, base, c, pl);
    pairs(o, v);
  };
  int half = 0, slot = 0;
  if (VEC)
    for (int i = 0; i < a.ahead; ++i) fetch(first + i, i);

  const unsigned slot0 = first_slot(a, kind, (unsigned)share);
  unsigned gate = 0, gate_end = 0;         // of a shared gate: the present row's, and the row after its last
  if (shared_gate && first < last) {
    gate = row_of(first) / a.per_gate;
    gate_end = (gate + 1) * a.per_gate;
  }
  // w_pre and e = w_post s, times a(g) of a shared gate
  auto make_e = [&](int c, f2 (&e)[4]) {
    f2 s[4];
    param(w_post, c, e);
    param(s_res, c, s);
#pragma unroll
    for (int k = 0; k < 4; ++k) e[k] = mul2(e[k], s[k]);
    if (shared_gate) {
      float g[8];
      load8<VEC>(g, row_at<TY>(gs, gate, a.ldg), c, pl);
      if (a.gate == BETTY_GATE_SIGMOID)
#pragma unroll
        for (int k = 0; k < 8; ++k) g[k] = sigmoid_gate<TX>(g[k]);
      pairs(s, g);
#pragma unroll
      for (int k = 0; k < 4; ++k) e[k] = mul2(e[k], s[k]);
    }
  };
  auto keep_e = [&](int c) {
    f2 e[4];
    make_e(c, e);
    sts16f(e_s + (2 * c) * G * 16, e[0].x, e[0].y, e[1].x, e[1].y);
    sts16f(e_s + (2 * c + 1) * G * 16, e[2].x, e[2].y, e[3].x, e[3].y);
  };
  auto coefficients = [&](int c, f2 (&w)[4], f2 (&e)[4]) {
    if constexpr (KEEP) {
      const float4 a0 = lds16f(w_s + (2 * c) * G * 16), a1 = lds16f(w_s + (2 * c + 1) * G * 16);
      const float4 b0 = lds16f(e_s + (2 * c) * G * 16), b1 = lds16f(e_s + (2 * c + 1) * G * 16);
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
      load8<VEC>(w, w_pre, c, pl);
      sts16f(w_s + (2 * c) * G * 16, w[0], w[1], w[2], w[3]);
      sts16f(w_s + (2 * c + 1) * G * 16, w[4], w[5], w[6], w[7]);
      if (bias) {
        float s[8];
        load8<VEC>(w, b_post, c, pl);
        load8<VEC>(s, s_res, c, pl);
        sts16f(b_s + (2 * c) * G * 16, w[0] * s[0], w[1] * s[1], w[2] * s[2], w[3] * s[3]);
        sts16f(b_s + (2 * c + 1) * G * 16, w[4] * s[4], w[5] * s[5], w[6] * s[6], w[7] * s[7]);
      }
      keep_e(c);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      accC[c][k] = accA[c][k] = both(0.f);
      if (GENERAL) {
        accD[c][k] = accB[c][k] = both(0.f);
        mask[c][k] = f2{inside<VEC>(pl, c, 2 * k) ? 1.f : 0.f, inside<VEC>(pl, c, 2 * k + 1) ? 1.f : 0.f};   // 0 outside the row
      }
    }
    if (shared_gate) {
      float zero[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        zero[k] = 0.f;
        if (G == 32) {
          sts4f(acc_s + (c * 8 + k) * G * 4, 0.f);
          if (GENERAL) sts4f(acc_s + (CH * 8 + c * 8 + k) * G * 4, 0.f);
        }
      }
      if (G > 32) {
        store_sums<VEC>(partials + d, zero, c, pl);
        if (bias) store_sums<VEC>(partials + 3 * (int64_t)d, zero, c, pl);
      }
    }
  }
  for (unsigned at = first; at < last; ++at) {
    row = row_of(at);
    if constexpr (VEC) {
      fetch(at + a.ahead, slot == 0 ? a.ahead : slot - 1);
      copies_wait(a.ahead);
      p = ring + slot * a.slot_bytes;
      slot = slot == a.ahead ? 0 : slot + 1;
      if (pl.shift) {
        if (has_u) { drop_head<TX>(p, pl); drop_head<TY>(p + at_u, pl); }
        if (has_o) drop_head<TX>(p + at_o, pl);
        if (has_y) drop_head<TY>(p + at_y, pl);
        if (row_gate) drop_head<TY>(p + at_g, pl);
      }
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
                for (int k = 0; k < 4; ++k) g[k] = f2{sigmoid_gate<TX>(g[k].x), sigmoid_gate<TX>(g[k].y)};
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
    // dX = dx' + r (dn0 - <dn>) + cn n with n = r (x - mean) and cn = -r <dn n>.  Every factor here is of the size of n, dn, x or
    // 1 / x: a coefficient of x itself would have r^3 in it, which leaves the fp32 range for rows beyond 1e-12 .. 1e12.
    float r = 1.f, q = 1.f, cn = 0.f, mean_dn = 0.f;
    if (a.pre != BETTY_NORM_NONE && has_u) {
      r = rsqrtf(fmaf(S[0], a.inv_d, a.eps));
      cn = -(r * (S[1] * a.inv_d)) * r;
      if (pre_layer) mean_dn = S[3] * a.inv_d;
    }
    float pm = 0.f;
    if (a.post != BETTY_NORM_NONE && has_y) {
      q = rsqrtf(fmaf(S[2], a.inv_d, a.eps));
      if constexpr (!GENERAL) pm = q * fmaf(r, S[NS - 2], fmaf(cn, r * S[NS - 1], S[3])) * a.inv_d;
    }
    const f2 r2 = both(r), cn2 = both(cn), q2 = both(q), pq2 = both(-pm * q), dn2 = both(-mean_dn);
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
          const f2 n = mul2(x[k], r2);
          dX[k] = fma2(n, cn2, dX[k]);
          f2 dn = mul2(u[k], w[k]);
          if (GENERAL) dn = add2(dn, dn2);          // subtracted before the scaling: r can be large where a row is flat
          dX[k] = fma2(dn, r2, dX[k]);
          if (GENERAL) {
            accD[c][k] = add2(accD[c][k], u[k]);
          }
          accC[c][k] = fma2(u[k], n, accC[c][k]);
        }
      }
      singles(out, dX);
      store8<VEC>(row_at<TX>(a.dx, row, a.lddx), out, c, pl);
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
          f2 b[4];
          if constexpr (KEEP) {
            const float4 b0 = lds16f(b_s + (2 * c) * G * 16), b1 = lds16f(b_s + (2 * c + 1) * G * 16);
            b[0] = f2{b0.x, b0.y}; b[1] = f2{b0.z, b0.w}; b[2] = f2{b1.x, b1.y}; b[3] = f2{b1.z, b1.w};
          } else {
            f2 s[4];
            param(b_post, c, b);
            param(s_res, c, s);
#pragma unroll
            for (int k = 0; k < 4; ++k) b[k] = mul2(b[k], s[k]);
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) z[k] = add2(b[k], z[k]);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) z[k] = mul2(z[k], dX[k]);
        if (a.gate == BETTY_GATE_SIGMOID)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            f2 s, n;
            sigmoid_gate<TX>(g[k].x, s.x, n.x);
            sigmoid_gate<TX>(g[k].y, s.y, n.y);
            g[k] = s;
            z[k] = mul2(z[k], mul2(s, n));
          }
        singles(out, z);
        store8<VEC>(row_at<TY>(a.dg, row, a.lddg), out, c, pl);
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
      if (!GENERAL) store8<VEC>(row_at<TY>(a.dy, row, a.lddy), out, c, pl);
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
          store8<VEC>(row_at<TY>(a.dy, row, a.lddy), out, c, pl);
        }
      }
    }
    if (has_y && shared_gate && (at + 1 == last || row + (unsigned)a.classes >= gate_end)) {           // the walker leaves the gate
      const unsigned g0 = gate * a.per_gate, g1 = min(gate_end, (unsigned)a.rows);
      const bool whole = a.classes == 1 && g0 >= first && g1 <= last;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float g[8], dg[8], w[8], s[8], b[8];
        load8<VEC>(g, row_at<TY>(gs, gate, a.ldg), c, pl);
        load8<VEC>(w, w_post, c, pl);
        load8<VEC>(s, s_res, c, pl);
        if (bias) load8<VEC>(b, b_post, c, pl);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float H = k & 1 ? accA[c][k / 2].y : accA[c][k / 2].x, E = !GENERAL ? 0.f : (k & 1 ? accB[GENERAL ? c : 0][k / 2].y : accB[GENERAL ? c : 0][k / 2].x);
          dg[k] = s[k] * (bias ? fmaf(b[k], E, w[k] * H) : w[k] * H);
          if (a.gate == BETTY_GATE_SIGMOID) {
            float n;
            sigmoid_gate<TX>(g[k], g[k], n);
            dg[k] *= g[k] * n;
          }
          if (G == 32) {
            const uint32_t at_a = acc_s + (c * 8 + k) * G * 4, at_b = at_a + CH * 8 * G * 4;
            sts4f(at_a, fmaf(g[k], H, lds4f(at_a)));
            if (GENERAL) sts4f(at_b, fmaf(g[k], E, lds4f(at_b)));
          } else {
            w[k] = g[k] * H;
            if (GENERAL) b[k] = g[k] * E;
          }
        }
        if (G > 32) {
          float was[8];
          load8<VEC>(was, partials + d, c, pl);
#pragma unroll
          for (int k = 0; k < 8; ++k) w[k] += was[k];
          store_sums<VEC>(partials + d, w, c, pl);
          if (bias) {
            load8<VEC>(was, partials + 3 * (int64_t)d, c, pl);
#pragma unroll
            for (int k = 0; k < 8; ++k) b[k] += was[k];
            store_sums<VEC>(partials + 3 * (int64_t)d, b, c, pl);
          }
        }
        if (whole) store_each<VEC>(row_at<TY>(a.dg, gate, a.lddg), dg, c, pl);
        else store_sums<VEC>(a.gate_partials + (int64_t)gate_slot(a, slot0, gate, g0 >= first, at) * d, dg, c, pl);
      }
      if (at + 1 < last) {
        gate = row_of(at + 1) / a.per_gate;
        gate_end = (gate + 1) * a.per_gate;
      }
#pragma unroll
      for (int c = 0; c < CH; ++c) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          accA[c][k] = both(0.f);
          if (GENERAL) accB[c][k] = both(0.f);
        }
        if constexpr (KEEP)
          if (at + 1 < last) keep_e(c);
      }
    }
  }
  if (shared_gate && G == 32)
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        accA[c][k] = f2{lds4f(acc_s + (c * 8 + 2 * k) * G * 4), lds4f(acc_s + (c * 8 + 2 * k + 1) * G * 4)};
        if (GENERAL) accB[c][k] = f2{lds4f(acc_s + (CH * 8 + c * 8 + 2 * k) * G * 4), lds4f(acc_s + (CH * 8 + c * 8 + 2 * k + 1) * G * 4)};
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
      if (G > 32) store_sums<VEC>(out, v, c, pl);
      else
#pragma unroll
        for (int k = 0; k < 8; ++k) combine[sub * W + (c * 8 + k) * 32 + t] = v[k];
    }
    if (G == 32) {
      __syncthreads();
      for (int j = threadIdx.x; j < d; j += blockDim.x) {
        float s = 0.f;
        for (int w = 0; w < subs; ++w) {              // column j is in another place in each class
          const int shift = VEC ? (int)(((blockIdx.x * subs + w) % a.classes * a.ld8) & 7) : 0, jj = j + shift;
          s += combine[w * W + (VEC ? (jj / 256 * 8 + jj % 8) * 32 + jj / 8 % 32 : j)];
        }
        out[j] = s;
      }
    }
  }
}

// Adds the blocks' column sums and forms the parameter gradients (the first param_blocks blocks: 32 columns each, SLICES
// slices of the list added in a fixed order), then the gates whose rows lie in several walkers' shares.
static constexpr int SLICES = 32, GATE_COLUMNS = 256;
// Every SLICES-th block's sums from block `slice` on, in order, U at a time: all of a batch's loads are on their way before the
// first is added, the last batch's too (left to the compiler that one became a load at a time: 2731 x 1537 fp32 6 us slower).
template <int NQ, int U>
__device__ __forceinline__ void add_blocks(float (&v)[4], const float* sums, int64_t d, int slice, int blocks) {
  for (int b = slice; b < blocks; b += U * SLICES) {
    float t[U][NQ];
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int k = 0; k < NQ; ++k) t[i][k] = b + i * SLICES < blocks ? sums[((int64_t)(b + i * SLICES) * NQ + k) * d] : 0.f;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int k = 0; k < NQ; ++k) v[k] += t[i][k];
  }
}
// SHARED: there are such gates (a kernel of its own, so that the others' sums keep their registers).
struct GateRows { int64_t n, i1, lo, hi; };       // of a class: its rows, the row after the gate's last, the shares that hold the gate's
template <typename TY, bool SHARED>
__global__ void __launch_bounds__(32 * SLICES) k_backward_sums(const Args a, int blocks, int param_blocks, float* __restrict__ dparams) {
  __shared__ float part[4][SLICES][32];
  pdl_enter();
  const int d = a.d;
  if (!SHARED || (int)blockIdx.x < param_blocks) {
    const int j = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5, nq = a.bias ? 4 : 2;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (j < d) {
      if (nq == 2) add_blocks<2, 10>(v, a.col_partials + j, d, slice, blocks);
      else add_blocks<4, 5>(v, a.col_partials + j, d, slice, blocks);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) part[i][slice][threadIdx.x & 31] = v[i];
    __syncthreads();
    if (slice < 4) {                 // one warp per quantity
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < SLICES; ++i) s += part[slice][i][threadIdx.x & 31];
      __syncwarp();
      part[slice][0][threadIdx.x & 31] = s;
    }
    __syncthreads();
    if (slice == 0 && j < d) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = part[i][0][threadIdx.x];
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
  int64_t gate = item;
  const int64_t gates = (a.rows + a.per_gate - 1) / a.per_gate;
  if (a.classes == 1 && gates >= a.shares) {      // more gates than shares: only the ones cut by the start of share item + 1 are open
    const int64_t cut = share_start(item + 1, a.rows, a.shares);
    gate = cut / a.per_gate;
    const int64_t g0 = gate * a.per_gate;
    if (g0 == cut || share_of(g0, a.rows, a.shares) != item) return;
  }
  const int64_t g0 = gate * a.per_gate, g1 = g0 + a.per_gate < a.rows ? g0 + a.per_gate : a.rows;
  constexpr int GS = 32 * SLICES / GATE_COLUMNS;
  __shared__ GateRows of_class[8];
  if ((int)threadIdx.x < a.classes) {             // once for the block: these are 64-bit divisions
    const int kind = threadIdx.x;
    const int64_t n = class_rows(a, kind), i0 = g0 > kind ? (g0 - kind + a.classes - 1) / a.classes : 0;
    const int64_t i1 = g1 > kind ? (g1 - kind + a.classes - 1) / a.classes : 0;
    of_class[kind] = i0 < i1 ? GateRows{n, i1, share_of(i0, n, a.shares), share_of(i1 - 1, n, a.shares)} : GateRows{0, 0, 0, -1};
  }
  __syncthreads();
  float s = 0.f;
  for (int kind = 0; kind < a.classes; ++kind) {
    const int64_t n = of_class[kind].n, i1 = of_class[kind].i1, lo = of_class[kind].lo, hi = of_class[kind].hi;
    if (hi < lo) continue;                        // the class has none of the gate's rows
    if (a.classes == 1 && lo == hi) return;       // one walker had all of the gate's rows and has written dg
    if (j < d) {
      int64_t w = lo + slice;
      if (slice == 0 && a.classes == 1) {         // the share that the gate begins in
        s = a.gate_partials[(int64_t)gate_slot(a, first_slot(a, kind, (unsigned)lo), (unsigned)gate, true, 0u) * d + j];
        w += GS;
      }
      if (n >= a.shares && !a.gate_sums.per_row) {
        const float* p = a.gate_partials + (int64_t)gate_slot(a, first_slot(a, kind, (unsigned)w), (unsigned)gate, false, 0u) * d + j;
        const int64_t step = (int64_t)GS * d * (a.classes == 1 ? 2 : 1);
#pragma unroll 8
        for (; w <= hi; w += GS, p += step) s += *p;
      } else {
        for (; w <= hi; w += GS) {
          const int64_t to = w == hi ? i1 : share_start(w + 1, n, a.shares);
          if (n < a.shares && share_start(w, n, a.shares) >= to) continue;       // an empty share: its place holds nothing
          s += a.gate_partials[(int64_t)gate_slot(a, first_slot(a, kind, (unsigned)w), (unsigned)gate, false, (unsigned)(to - 1)) * d + j];
        }
      }
    }
  }
  float* sums = &part[0][0][0];
  sums[slice * GATE_COLUMNS + lane] = s;
  __syncthreads();
  if (slice == 0 && j < d) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < GS; ++i) s += sums[i * GATE_COLUMNS + lane];
    row_at<TY>(a.dg, gate, a.lddg)[j] = from_f<TY>(s);
  }
}

// Blocks of the grid, and shares of each class: as many thread groups as the device holds, at most one per row, at least one
// per class.
void backward_grid(int64_t rows, const Layout& l, int classes, int& blocks, int& shares) {
  const int groups = l.threads / l.G;
  const int64_t walkers = (int64_t)current_sm_count() * l.blocks_per_sm * groups, most = (rows + classes - 1) / classes;
  int64_t n = walkers / classes;
  if (n > most) n = most;
  if (n < 1) n = 1;
  shares = (int)n;
  blocks = (int)((n * classes + groups - 1) / groups);
}
GateSums gate_sums_of(int64_t rows, int64_t per_gate, int classes, int shares) {
  if (classes == 1) return {2 * (int64_t)shares, 2, 0, 0, 1};
  const int64_t pairs = shares + (rows + per_gate - 1) / per_gate, most = (rows + classes - 1) / classes;
  if (most < pairs) return {most, 0, 0, 1, 0};
  return {pairs, 1, 1, 0, 0};
}
static inline bool is_general(int bias, int pre, int post) { return bias || pre == BETTY_NORM_LAYER || post == BETTY_NORM_LAYER; }
// chunks per thread of the wide kernel: the layer norms' and biases' sums leave registers for one
static constexpr int backward_chunks(bool general) { return general ? 1 : 2; }
Layout backward_layout(const betty_block_norm_cfg* c, int64_t rows, int xd, int yd, int classes) {
  const bool gated = c->gate != BETTY_GATE_NONE, general = is_general(c->bias, c->pre, c->post);
  const bool row_gate = gated && c->rows_per_gate == 1;             // a gate shared by rows stays in L1
  Needs n = {2, row_gate ? 3 : 2, backward_chunks(general), 1, 0, 0};
  n.kept_arrays = general ? 3 : 2;                                                                    // w_pre, e (, b s)
  n.sum_arrays = gated && !row_gate && c->d <= 32 * 8 * MAX_CH ? (general ? 2 : 1) : 0;               // A (, B) where a warp holds a row
  Layout l = layout_of(c->d, rows, xd, yd, classes, n);
  const size_t combine = l.G == 32 ? (size_t)(l.threads / 32) * l.chunks * 256 * sizeof(float) : 0;
  if (l.smem < combine) l.smem = combine;
  return l;
}

template <typename TX, typename TY, bool VEC, int CH, bool GENERAL, bool SHARED>
static betty_status launch_backward(cudaStream_t stream, const Args& a, const Layout& l, float* dparams) {
  static SmemLimit limit = {};
  if (l.smem > 40 * 1024) BETTY_TRY(ensure_dynamic_smem(k_backward<TX, TY, VEC, CH, GENERAL, SHARED>, limit, l.smem));
  int blocks, shares;
  backward_grid(a.rows, l, a.classes, blocks, shares);
  launch_pdl(k_backward<TX, TY, VEC, CH, GENERAL, SHARED>, dim3(blocks), dim3(l.threads), l.smem, stream, a);
  BETTY_LAUNCH_CHECK();
  const int param_blocks = (a.d + 31) / 32;
  int64_t items = 0;
  if (SHARED) {
    const int64_t gates = (a.rows + a.per_gate - 1) / a.per_gate;
    items = a.classes > 1 || gates < a.shares ? gates : a.shares - 1;
  }
  launch_pdl(k_backward_sums<TY, SHARED>, dim3((unsigned)(param_blocks + items * ((a.d + GATE_COLUMNS - 1) / GATE_COLUMNS))), dim3(32 * SLICES), 0, stream, a,
             blocks, param_blocks,
             dparams);
  BETTY_LAUNCH_CHECK();
  return BETTY_OK;
}
template <typename TX, typename TY, bool GENERAL, bool SHARED>
static betty_status backward_shape(cudaStream_t stream, const Args& a, const Layout& l, float* dparams) {
  if (!l.vec) return launch_backward<TX, TY, false, 4, GENERAL, SHARED>(stream, a, l, dparams);
  return l.chunks == 1 ? launch_backward<TX, TY, true, 1, GENERAL, SHARED>(stream, a, l, dparams)
                       : launch_backward<TX, TY, true, 2, GENERAL, SHARED>(stream, a, l, dparams);
}
template <typename TX, typename TY, bool GENERAL>
static betty_status backward_gated(cudaStream_t stream, const Args& a, const Layout& l, float* dparams) {
  const bool shared = a.gate != BETTY_GATE_NONE && a.per_gate > 1;
  return shared ? backward_shape<TX, TY, GENERAL, true>(stream, a, l, dparams) : backward_shape<TX, TY, GENERAL, false>(stream, a, l, dparams);
}
template <typename TX, typename TY>
static betty_status backward_typed(cudaStream_t stream, const Args& a, const Layout& l, float* dparams) {
  return is_general(a.bias, a.pre, a.post) ? backward_gated<TX, TY, true>(stream, a, l, dparams) : backward_gated<TX, TY, false>(stream, a, l, dparams);
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
