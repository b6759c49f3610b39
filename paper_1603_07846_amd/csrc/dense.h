// dense.h -- products of dense matrices with their epilogues, and the small
// kernels around them: the launchers behind include/singa_mi_dense.h.  Like
// internal.h, everything here takes arguments that the ABI layer has checked.
#pragma once

#include "internal.h"

namespace singa {

enum Act { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_SILU = 3 };

// What a product does with its sum over k, element (row, col) of M x N.
//   EPI_OUT     v = alpha sum + bias[col]; z = v (kept when z is given);
//               y = act(v) + res, or y += that (add, fp32 outputs), zeroed in
//               rows without a valid label (labels given)
//   EPI_LSE     the maximum and the sum of exponentials of v = sum + bias[col]
//               over each STAT_COLS columns, and v at the row's label: the
//               logits themselves are not stored
//   EPI_DLOGITS softmax(v) by lse[row] - [col is the row's label] in rows with a
//               valid label, else 0, stored in the product's type (and, with
//               more, what that rounding left).  The factor scale / count of the
//               loss is left to the products that take these (alpha), so that
//               a label's entry, nearly -1, is stored nearly exactly: with the
//               factor in it, its rounding was the same for every row and put
//               0.3 % on all of dx.
enum Epi { EPI_OUT = 0, EPI_LSE = 1, EPI_DLOGITS = 2 };

constexpr int STAT_COLS = 64;

struct Epilogue {
  const float* alpha = nullptr;  // one value
  const float* bias = nullptr;  // [N]
  int act = ACT_NONE;
  const void* res = nullptr;  // T [M][N]
  void* z = nullptr;          // T [M][N]
  void* y = nullptr;          // T or fp32 [M][ldy]
  long ldy = 0;
  int out_f32 = 0, add = 0;
  // loss: labels counted from column col0 of this product
  const int32_t* labels = nullptr;
  int classes = 0;  // a label is valid in [0, classes)
  int col0 = 0;
  float2* stats = nullptr;  // [M][nstat] (maximum, sum), column group stat0 + ...
  int nstat = 0, stat0 = 0;
  float* zlab = nullptr;       // [M]
  const float2* lse = nullptr;  // [M], as row_lse makes them
  bf16_t* more = nullptr;  // the further terms (see TERMS), one behind the other
  int rows_padded = 0;  // dlogits rows from M up to here are zeroed (a sum over two halves reads them)
  float* colsum = nullptr;  // [row groups][N]: sums of the dlogits over COLSUM_ROWS rows
};

constexpr int COLSUM_ROWS = 64;

// An operand: logical rows x K.  kc: stored row by row (K contiguous, ld
// elements from row to row); otherwise stored k by k (rows contiguous, ld
// elements from k to k).  The stored rows start at 16-byte boundaries, and
// what lies between their end and the next such boundary is zero.
struct Operand {
  const void* p;
  long ld;
  bool kc;
};

// y (M x N) = epilogue(A B^T), A: M x K, B: N x K.
struct Product {
  int dt = BF16;
  int M = 0, N = 0, K = 0;
  Operand a{}, b{};
  // a k index from `wrap` on continues in A and starts again in B, and so from
  // 2 wrap on: A's terms one behind the other, each with the same B.  A
  // multiple of K_TILE elements; 0: one term.  K counts all terms.
  int wrap = 0;
  int kb = 0;  // k rows that B has (0: K)
  int epi = EPI_OUT;
  Epilogue e;
  bool raw = false;  // see product_splits
  const char* name = "";
  double flops = 0;
};

// An fp32 gradient of bf16 weights takes a computed dz (fp32) in this many
// bf16 terms, each the rounding of what the ones before left: 3 x 8 bits of
// significand hold all of fp32's 24.  (Two, an error of 2^-18 at most, put
// 1.2e-6 on dw where the fp32 sums alone leave 0.3e-6; one 1.6e-3.)  It triples
// that product (4000 x 4096 x 4096, GELU: 298 us where one term takes 110, the
// whole call 457 and 261; the loss of 4096 x 2048 x 100000: 8650 and 5780).
//
// A bf16 result, dx or a bf16 dw, takes one term: dz rounded once.  Its own
// rounding is as large (relative error of all gradients of that GELU layer
// 0.0023 so, 0.0017 with an unrounded dz; of the loss 0.0018 and 0.0017 at 256
// x 4096 x 1000, 0.0017 both at 4096 x 2048 x 100000), and every further term
// is one more product (dx of 4000 x 4096 over 4096 / 8192 / 12288: 118 / 204 /
// 297 us).
constexpr int TERMS = 3;

constexpr int K_TILE = 64;  // a multiple of every kernel's K-tile

// Workspace for the partial sums of a product whose tiles cannot fill the GPU.
size_t product_partial_bytes(int dt, int M, int N, int K, int epi);
hipError_t launch_product(const Product& p, float* partial, hipStream_t st);
// The products of a layer's source gradient (A K contiguous, B rows
// contiguous) and weight gradient (both rows contiguous), in one launch where
// that is faster; workspace: the larger of the two products' and this.
size_t pair_partial_bytes(int dt, int Ma, int Na, int Ka, int Mb, int Nb, int Kb);
// sums, finish (may be null): done by further workgroups of that launch, or before.
struct ColumnSums;
struct LossFinish;
hipError_t launch_pair(const Product& dx, const Product& dw, const ColumnSums* sums, const LossFinish* finish, float* partial,
                       hipStream_t st);
// Number of partial sums of that product; launch_product with `raw` writes
// them ([M][N rounded up to 8] each, also when it is one) and stops there.
int product_splits(int dt, int M, int N, int K);

// Whether launch_skinny is the faster one (copied: operands for the tiles are
// needed anyway).
bool product_skinny(int dt, int M, int N, int K, bool copied);
// The same product for few rows (M <= SKINNY_ROWS), A and B both K contiguous
// with ld = K, any alignment.  EPI_OUT and EPI_LSE (STAT_COLS
// of SKINNY_COLS columns).
constexpr int SKINNY_ROWS = 512, SKINNY_COLS = 16;
hipError_t launch_skinny(const Product& p, hipStream_t st);

// Zeros, by a kernel (a captured memset node is not replayed reliably).
hipError_t launch_zero(void* p, size_t bytes, hipStream_t st);
// out [rows][ldo] = in [rows][cols], zero from cols to ldo; rows without a
// valid label (labels given) become zero.
hipError_t launch_pack(int dt, const void* in, void* out, long rows, int cols, long ldo, const int32_t* labels,
                       int classes, hipStream_t st);
// Two matrices of equal row length at once (no labels).
hipError_t launch_pack2(int dt, const void* in, void* out, long rows, const void* in2, void* out2, long rows2, int cols,
                        long ldo, hipStream_t st);
// dz = dy act'(z) as T [rows_padded][ldz] (zero past rows and cols), more (may
// be null) its further terms, colsum [ceil(rows / dact_rows())][cols] (may be
// null) the sums of the unrounded dz; dz may be null.
int dact_rows(long rows, int cols);  // rows per workgroup
hipError_t launch_dact(int dt, int act, const void* dy, const void* z, void* dz, void* more, float* colsum, long rows,
                       long rows_padded, int cols, long ldz, hipStream_t st);
// out[c] (+)= alpha (null: 1) times the sum of src[0 .. rows - 1][c], in a fixed
// order; SUM_COLS columns per workgroup of 256 threads
constexpr int SUM_COLS = 16;
struct ColumnSums {
  const void* src;  // [rows][cols] of type dt
  int dt;
  long rows;
  int cols;
  float* out;
  int add;
  const float* alpha;
};
inline unsigned sums_wgs(const ColumnSums& s) { return (unsigned)((s.cols + SUM_COLS - 1) / SUM_COLS); }
hipError_t launch_column_sums(const ColumnSums& s, hipStream_t st);
// out (T [rows][cols]) = in (fp32 [rows][cols]), zero in rows without a valid label
hipError_t launch_round_rows(int dt, const float* in, void* out, long rows, int cols, const int32_t* labels,
                             int classes, hipStream_t st);
// stats [rows][nstat], zlab -> lse[row] (may be null), loss[1 + row]
hipError_t launch_lse(const float2* stats, int nstat, const float* zlab, const int32_t* labels, int classes, long rows,
                      float2* lse, float* loss, hipStream_t st);
// loss[0] = mean of loss[1 ..] over the counted rows, unit = scale / count (0 when none; may be null)
hipError_t launch_loss_mean(const int32_t* labels, int classes, long rows, float* loss, float* unit, float scale,
                            hipStream_t st);
// The same two at once, for few rows: one workgroup goes through them, row by
// row (LSE_FINISH_ROWS of any length) or a wave per row, eight rounds at most
// (a launch less: 13 x 64 x 7817 18 -> 15 us).
constexpr int LSE_FINISH_ROWS = 4;
inline bool lse_finish_pays(int rows, int nstat) {
  return rows <= LSE_FINISH_ROWS || (long)((rows + 15) / 16) * ((nstat + 63) / 64) <= 8;
}
hipError_t launch_lse_finish(const float2* stats, int nstat, const float* zlab, const int32_t* labels, int classes, int rows,
                             float* loss, hipStream_t st);
// Rows of kept logits: z holds `splits` partial sums [rows][ldz] of them (the
// bias not added).  Written: loss[1 + row]; unless dz is null the dlogits as
// EPI_DLOGITS makes them (T [rows_padded][ldd], zero past rows and classes)
// and their further terms (more); with keep_dz their unrounded values into
// the first [rows][ldz] of z (rows with a valid label only); unless xc is null
// the rows of x as launch_pack makes them with labels.
struct LossRows {
  float* z;
  long ldz;
  int splits;
  const float* bias;
  const int32_t* labels;
  long rows, rows_padded;
  int classes;
  float* loss;
  void *dz, *more;
  long ldd;
  int keep_dz;
  const void* x;
  void* xc;
  int in;
  long ldx;
  float2* stats;  // [rows][loss_parts(classes)]: several workgroups per row; null: one
  float* unit;    // unless null, scale / count is written there (up to FINISH_ROWS rows)
  float scale;
};
constexpr int LOSS_PART = 4096;  // classes per workgroup then
inline int loss_parts(int classes) { return (classes + LOSS_PART - 1) / LOSS_PART; }
hipError_t launch_loss_rows(int dt, const LossRows& a, hipStream_t st);
// The mean of up to FINISH_ROWS rows and, unless db is null, db (+)= scale /
// count times the sum of the valid rows of dz.  Beside the gradients' products
// and by launches of their own, us for loss and gradients of 256 inputs: bf16
// 32 x 1000 classes 26 / 32, 256 x 1000 27 / 41, 256 x 10000 59 / 64, 900 x 1000
// 41 / 55, 900 x 10000 122 / 118, 1500 x 1000 47 / 57, 1500 x 10000 183 / 164,
// 3000 x 1000 76 / 64; fp32 900 x 1000 53 / 66, 1500 x 1000 62 / 75, 1500 x
// 10000 333 / 360, 3000 x 1000 91 / 104, 6000 x 1000 186 / 154.
constexpr int FINISH_ROWS = 1024, FINISH_COLS = 8;
struct LossFinish {
  const int32_t* labels;
  int classes, rows;
  float* loss;
  float scale;
  const float* dz;
  long ld;
  float* db;
  int add;
};
inline unsigned finish_wgs(const LossFinish& f) { return f.db ? (unsigned)((f.classes + FINISH_COLS - 1) / FINISH_COLS) : 1u; }
hipError_t launch_loss_finish(const LossFinish& f, hipStream_t st);
// colsum [groups][cols] of dzf [rows][ld] over COLSUM_ROWS rows each, those
// with a valid label
hipError_t launch_colsum_rows(const float* dzf, long ld, float* colsum, long rows, int cols, const int32_t* labels,
                              int classes, hipStream_t st);

}  // namespace singa
