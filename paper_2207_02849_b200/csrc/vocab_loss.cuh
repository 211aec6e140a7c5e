// Losses of a language model over its vocabulary (vocab_loss.cu: rows, statistics and the C entries; vocab_products.cu: the
// matrix products).
//
//   z_iv = x_i . w_v / T,   lse_i = log sum_v exp z_iv,   q_iv = exp(z_iv - lse_i)
//   cross entropy   l_i = (1 - e) (lse_i - z_it) + e (lse_i - mean_v z_iv) + zeta lse_i^2
//   distillation    l_i = sum_j p_ij (log p_ij - z_i,id(j) + lse_i),   p_i = softmax of the teacher's entries / T
//   both            dl_i/dz_iv = a q_iv + b - sum over the row's entries at v of p,   a = 1 + 2 zeta lse_i, b = -e / V
//                   dx_i = (g_i / T) sum_v dz_iv w_v,   dw_v = sum_i (g_i / T) dz_iv x_i
//
// The entries of a row are (id, p) pairs in ascending order of id: one, (t, 1 - e), of a cross entropy.  Rows that do not
// count (and, in a backward pass, rows with g = 0) are left out before the products: the others are copied one after the
// other into the workspace, on 16-byte boundaries, so that what a row left out holds reaches nothing and costs nothing, and
// the host needs no count.  Logarithms and exponentials are taken to the base 2: y = z log2(e), lse2 = lse log2(e).
#pragma once
#include "tensor_core.cuh"

namespace betty {
namespace vocab {

static constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
static constexpr int MAX_TOP = 1024;
static constexpr int NO_ID = 0x7FFFFFFF;       // an entry that is none

struct RowCoef { float lse2, a, b, e; };       // dz = a 2^(y - lse2) + b - e p, as it is stored for the products
struct Meta {
  int32_t n;             // rows that count
  int32_t split;         // parts of the contraction of dX, each with its own sums
  float dw_scale;        // what a sum over the stored dz and x is multiplied by to give dW
};

// What the products need to know of one call.
struct Shape {
  int dtype;             // operands
  int rows;              // upper bound of the rows that count
  int64_t rpad;          // rows of the workspace's matrices, a multiple of 256
  int vocab, d;
  int64_t dp;            // d rounded up to a multiple of 64: leading dimension of the workspace's copies of x
  float c2;              // log2(e) / T
  int top;               // entries of a row
  int pairs;             // logits: pairs of SMs take tiles of 256 x 256, else an SM takes 128 x width
  int width;
  int product_pairs;     // gradients: the same choice
  int piece;             // columns of the vocabulary at a time (backward), a multiple of 256
  int twice;             // gradients of up to TWICE_ROWS rows: see there
  int64_t sum_rows;      // rows of dX's sums: room for `split` times the rows that count
  int want_dx, want_dw;
};

// The gradients' coefficients are rounded to the operands' type.  With so few rows that half of a contraction chunk over them is empty, what the
// rounding took away is kept as rows of its own, this many behind the rounded ones (and the copies of x twice), and goes through
// the same products, and the results are as near as their own last rounding (24 rows x 32000 x 2048, dX and dW in bf16 against 64
// bits: 2.4e-3 -> 1.7e-3, for 93 -> 96 us).  Room for 64 rows, in a second chunk, would do the same for 33 to 64 rows (2.4e-3 -> 1.7e-3, fp16
// 3.1e-4 -> 2.1e-4), but not for nothing: 33, 48 and 64 rows take 93 us as they are and 107 to 108 with it, and fewer rows 108 instead of 96.
static constexpr int TWICE_ROWS = 32;

// ---- how the tiles of the gradients' products are spread ----
// dX's tiles contract over the piece's columns, dW's over the rows: their lengths differ, by much where there are few rows.
struct Products {
  int row_tiles, d_tiles, col_tiles;   // tiles along the rows, d and the piece's columns
  int dx_chunks, dw_chunks;            // lengths of the contractions
};
__host__ __device__ inline Products products_of(int n, int d, int cols, int lanes) {
  return {(n + lanes - 1) / lanes, (d + lanes - 1) / lanes, (cols + lanes - 1) / lanes, (cols + tc::BK - 1) / tc::BK, (n + tc::BK - 1) / tc::BK};
}
// A tile's time in contraction chunks, of 0.34 us in a pair: four more until the first copies are there and the last sums stored, and a
// tile of dW takes the time of four at least, in which it is stored.
__host__ __device__ inline int dx_cost(const Products& p, int split) { return (p.dx_chunks + split - 1) / split + 4; }
__host__ __device__ inline int dw_cost(const Products& p) { return (p.dw_chunks > 4 ? p.dw_chunks : 4) + 1; }

struct Buffers {
  Meta* meta;
  int32_t* src;          // [rpad] row of the caller's that row i of the copies is
  int32_t* pos;          // [rows] where a row went, -1: left out
  uint16_t* x;           // [rpad, dp]
  uint16_t* x_dw;        // [rpad, dp] as the gradient of W takes it (fp16: scaled, else x itself)
  int2* entry;           // [top][rpad] entries of the rows that count, the next row's beside a row's: id, and the bits of p
  int2* entry_in;        // [rows, top] the same of all rows (distillation)
  float2* part;          // [parts][rpad] maximum and sum of 2^(y - maximum) of a part of a row
  float* part_y;         // [parts][rpad] sum of y (smoothing only)
  float* y_entry;        // [top][rpad] y at the entries
  RowCoef* coef;         // [rpad]
  float* row_scale;      // [rpad] what a row of dX is multiplied by
  uint16_t* dz;          // [rpad, piece]; twice: rows from TWICE_ROWS on are the remainders
  float* dx;             // [split][rows that count, up to whole tiles; dp], sum_rows in all
  StatusBlock* sb;
};

// A forward pass over few rows that start on 16-byte boundaries: x is read in place, and which rows count is looked at where their losses
// are made (rows left out make statistics that nothing reads).  8 rows x 32000 x 1024 21.7 -> 17.6 us.
struct InPlace {
  const void* x; int64_t ldx;
  const void* target; int id64; float share;   // cross entropy: an entry (target, share) per row; else Buffers::entry, a row each
};
static constexpr int IN_PLACE_ROWS = 128;

int logits_parts(const Shape& s);
// part, part_y (if not null) and y_entry of all rows that count (in_place: of all rows); w_ahead: w is not written by the kernels of this
// call
betty_status logits_statistics(cudaStream_t stream, const Shape& s, const Buffers& b, const tc::Operand& w, bool w_ahead, const InPlace* in_place);
// dX's fp32 sums (want_dx) and dW (dw not null), piece by piece
betty_status logits_gradients(cudaStream_t stream, const Shape& s, const Buffers& b, const tc::Operand& w, bool w_ahead, void* dw, int64_t lddw, int dw_dtype);
void choose_shape(Shape& s, bool backward);

}  // namespace vocab
}  // namespace betty
