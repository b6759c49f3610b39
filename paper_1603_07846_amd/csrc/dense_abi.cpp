// dense_abi.cpp -- the C entry points declared in include/singa_mi_dense.h:
// argument checks, workspace carving and the order of the kernels.  Nothing is
// enqueued unless every check passes.
#include "singa_mi_dense.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <memory>
#include <new>

#include "dense.h"
#include "gradnorm.h"

using namespace singa;

namespace {

inline int status(hipError_t e) { return e == hipSuccess ? SINGA_OK : SINGA_ERR_HIP; }
inline bool aligned_to(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
inline long up(long v, long a) { return (v + a - 1) / a * a; }
inline int vec(int dt) { return dt == BF16 ? 8 : 4; }
bool dtype_ok(int dt) { return dt == SINGA_F32 || dt == SINGA_BF16; }

constexpr int kMaxFeatures = 1 << 20;  // a row stays below 2^23 bytes, so 256 of them have 32-bit offsets

constexpr int kMaxRows = 1 << 28;
constexpr long kMaxMatrix = 1L << 37;  // elements of a matrix (or rows x classes): tiles and workgroups stay below 2^24

// Hands out 256-byte aligned parts of a workspace (or, from NULL, counts them;
// the first 256 bytes make up for a base that is only 16-byte aligned).
struct Carver {
  char* base;
  size_t used = 0;
  explicit Carver(void* p) : base((char*)(((uintptr_t)p + 255) & ~(uintptr_t)255)) {}
  void* take(size_t bytes) {
    void* p = base + used;
    used += (bytes + 255) & ~(size_t)255;
    return bytes ? p : nullptr;
  }
  template <typename T> T* take(size_t n) { return (T*)take(n * sizeof(T)); }
  size_t bytes() const { return used ? used + 256 : 0; }
};

int check_ws(const void* ws, size_t have, size_t need) {
  if (!need) return SINGA_OK;
  if (!ws || have < need) return SINGA_ERR_WORKSPACE;
  return aligned_to(ws, 16) ? SINGA_OK : SINGA_ERR_ALIGN;
}

int shape(int rows, int in, int out) {
  if (rows < 0 || in < 1 || out < 1) return SINGA_ERR_SHAPE;
  if (in > kMaxFeatures || out > kMaxFeatures || rows > kMaxRows) return SINGA_ERR_UNSUPPORTED;
  if ((long)rows * in > kMaxMatrix || (long)rows * out > kMaxMatrix || (long)in * out > kMaxMatrix) return SINGA_ERR_UNSUPPORTED;
  return SINGA_OK;
}

// What a call reads or writes (NULL: nothing).
struct Span {
  const void* p;
  size_t bytes;
};
bool apart(const Span& a, const Span& b) {
  const uintptr_t pa = (uintptr_t)a.p, pb = (uintptr_t)b.p;
  return !a.p || !b.p || pa + a.bytes <= pb || pb + b.bytes <= pa;
}
// Workgroups write outputs while others still read: no output, and no
// workspace, may share memory with an input or another output.
template <int O, int I> int check_apart(const Span (&outs)[O], const Span (&ins)[I]) {
  for (int i = 0; i < O; ++i) {
    for (int j = 0; j < i; ++j)
      if (!apart(outs[i], outs[j])) return SINGA_ERR_UNSUPPORTED;
    for (const Span& in : ins)
      if (!apart(outs[i], in)) return SINGA_ERR_UNSUPPORTED;
  }
  return SINGA_OK;
}
Span span(const void* p, long rows, long cols, int dt) { return {p, (size_t)rows * cols * dt_size(dt)}; }
Span ws_span(const void* ws, size_t need) { return {need ? ws : nullptr, need}; }

// The row length of a matrix kept in the workspace: rows a multiple of 4 KB
// apart would all start in the same memory channel (a product over 32768 of k:
// 530 us, with 64 elements more per row 443).
long padded_row(long cols, size_t es) {
  const long ld = up(cols, 8);
  return ld * es % 4096 == 0 ? ld + 64 : ld;
}

// An operand's row length in a form that the tiles take.
struct Packed {
  long ld;
  bool copy;
};
Packed packed(int dt, int cols) {
  const long ld = up(cols, vec(dt));
  return {ld, ld != cols};
}

// ---------------------------------------------------------------- forward
struct FwdWs {
  bool skinny;
  Packed k;
  void *xp, *wp;
  float* partial;
};

size_t carve_fwd(int dt, int rows, int in, int out, void* ws, FwdWs* o) {
  Carver c(ws);
  *o = FwdWs{};
  o->skinny = product_skinny(dt, rows, out, in, false);
  if (rows == 0 || o->skinny) return 0;
  const size_t es = dt_size(dt);
  o->k = packed(dt, in);
  o->xp = c.take(o->k.copy ? (size_t)rows * o->k.ld * es : 0);
  o->wp = c.take(o->k.copy ? (size_t)out * o->k.ld * es : 0);
  o->partial = (float*)c.take(product_partial_bytes(dt, rows, out, in, EPI_OUT));
  return c.bytes();
}

// ---------------------------------------------------------------- backward
// Partial sums of the gradients' products, dx (rows x in over out) and dw (out
// x in over kw), by themselves or together.
size_t gradient_partial_bytes(int dt, int rows, int in, int out, int kw) {
  return std::max({product_partial_bytes(dt, rows, in, out, EPI_OUT), product_partial_bytes(dt, out, in, kw, EPI_OUT),
                   pair_partial_bytes(dt, rows, in, out, out, in, kw)});
}

struct BwdWs {
  Packed k;
  long ldz, rows_padded, groups;
  bool own_dz, split;  // dz in the workspace; in TERMS terms
  void *dz, *more, *xp, *wp;
  float *colsum, *partial;
};

size_t carve_bwd(int dt, int rows, int in, int out, int act, int dw_dt, void* ws, BwdWs* o) {
  Carver c(ws);
  *o = BwdWs{};
  if (rows == 0) return 0;
  const size_t es = dt_size(dt);
  o->k = packed(dt, in);
  const Packed n = packed(dt, out);
  o->split = dt == BF16 && dw_dt == F32 && (act == ACT_GELU || act == ACT_SILU);
  o->own_dz = act != ACT_NONE || n.copy;
  o->ldz = o->own_dz ? padded_row(out, es) : out;
  o->rows_padded = o->split ? up(rows, K_TILE) : rows;
  const size_t half = (size_t)o->rows_padded * o->ldz;
  o->dz = c.take(o->own_dz ? half * (o->split ? TERMS : 1) * es : 0);
  o->more = o->split ? (char*)o->dz + half * es : nullptr;
  o->xp = c.take(o->k.copy ? (size_t)rows * o->k.ld * es : 0);
  o->wp = c.take(o->k.copy ? (size_t)out * o->k.ld * es : 0);
  o->groups = (rows + dact_rows(rows, out) - 1L) / dact_rows(rows, out);
  o->colsum = c.take<float>(o->groups * (size_t)out);
  const int kw = (int)(o->rows_padded * (o->split ? TERMS : 1));
  o->partial = (float*)c.take(gradient_partial_bytes(dt, rows, in, out, kw));
  return c.bytes();
}

// ------------------------------------------------------------------- loss
// Logits of up to kKeep bytes (fp32) are kept between the two passes, larger
// ones are formed twice, kPiece bytes of dlogits (a term) at a time.  Kept /
// formed twice, us for loss and gradients of 1024 inputs, rows x classes:
//   fp32  256 x 1000 51 / 123, 256 x 16000 253 / 310, 512 x 32000 872 / 1032,
//         1024 x 32000 1739 / 2010, 4096 x 32000 6684 / 7885: keeping is faster
//         throughout, and the limit is what the workspace may cost
//   bf16  256 x 1000 30 / 46, 256 x 4000 47 / 60, 256 x 8000 (8 MB) 72 / 74, 512 x
//         16000 169 / 157, 512 x 32000 299 / 258, 1024 x 32000 650 / 464, 4096 x
//         32000 2074 / 1569, with 4096 inputs 2048 x 32000 2628 / 2663: the
//         product is cheap beside the traffic of fp32 logits, and from 8 MB up
//         to the limit keeping costs up to 16 %, with few inputs more (128
//         inputs, 512 x 32000 175 / 92; 256, 2000 x 4000 102 / 79)
// The loss alone: bf16 256 x 1000 16 / 16, with 4096 inputs 21 / 37; 512 x 16000 44
// / 28; fp32 512 x 16000 148 / 133, 256 x 4000 34 / 75.
// Pieces of 128 / 256 / 1024 MiB, bf16: 4096 x 2048 x 100000 8781 / 8733 / 8950
// us, 2048 x 1024 x 200000 5551 / 5065 / 5053, 8192 x 1024 x 50000 5199 / 4944 /
// 5556; fp32 4096 x 512 x 100000 12840 / 12538 / 13073.
constexpr size_t kKeep = 64u << 20;
constexpr size_t kPiece = 256u << 20;

struct LossWs {
  Packed k;
  bool keep, skinny, split, one;  // logits kept; few rows; dlogits in TERMS terms; one piece
  long ldd, rows_padded, piece;   // dlogits: row length, rows; classes per piece
  int nstat, splits;  // splits, ldl: partial sums of kept logits and their row length
  long ldl;
  void *dz, *more, *xc, *xp, *wp;
  float *unit, *zlab, *logits, *dxf, *colsum, *partial;
  float2 *stats, *lse;
};

size_t carve_loss(int dt, int rows, int in, int classes, bool grad, int dw_dt, void* ws, LossWs* o) {
  Carver c(ws);
  *o = LossWs{};
  if (rows == 0) return 0;
  const size_t es = dt_size(dt);
  o->k = packed(dt, in);
  // (the loss of a few rows alone takes two launches that way, four after tiles)
  o->skinny = product_skinny(dt, rows, classes, in, grad) || (!grad && rows <= LSE_FINISH_ROWS);
  o->ldl = up(classes, 8);
  o->keep = (!o->skinny || grad) && (size_t)rows * o->ldl * 4 <= kKeep;
  o->split = grad && dt == BF16 && dw_dt == F32;
  o->rows_padded = o->split ? up(rows, K_TILE) : rows;
  // copies for the tiles
  const bool tiles = !o->skinny || grad;
  o->wp = c.take(tiles && o->k.copy ? (size_t)classes * o->k.ld * es : 0);
  o->xp = c.take(tiles && o->k.copy ? (size_t)rows * o->k.ld * es : 0);
  size_t partial = 0;
  if (o->keep) {
    o->splits = o->skinny ? 1 : product_splits(dt, rows, classes, in);
    o->logits = c.take<float>((size_t)o->splits * rows * o->ldl);
    // rows that do not fill the chip, and several parts of each (in two launches:
    // 64 x 50000 bf16 86 us against 107 with a workgroup per row, fp32 137
    // against 155; at 10000 classes 43 against 40, and from 256 rows on 60
    // against 53, 500 x 30000 177 against 172)
    o->stats = rows < 512 && classes > 2 * LOSS_PART ? c.take<float2>((size_t)rows * loss_parts(classes)) : nullptr;
  } else {
    o->nstat = (classes + (o->skinny ? SKINNY_COLS : STAT_COLS) - 1) / (o->skinny ? SKINNY_COLS : STAT_COLS);
    o->stats = c.take<float2>((size_t)rows * o->nstat);
    o->zlab = c.take<float>(rows);
    o->lse = c.take<float2>(rows);
  }
  if (grad) {
    o->unit = c.take<float>(1);
    // whole tiles of classes per piece
    long piece = (long)(kPiece / es) / o->rows_padded / 256 * 256;
    if (piece < 256) piece = 256;
    o->one = o->keep || piece >= classes;
    o->piece = o->one ? classes : piece;
    o->ldd = padded_row(o->piece, es);
    const size_t half = (size_t)o->rows_padded * o->ldd;
    o->dz = c.take(half * es * (o->split ? TERMS : 1));
    o->more = o->split ? (char*)o->dz + half * es : nullptr;
    o->xc = c.take((size_t)rows * o->k.ld * es);
    o->dxf = o->one ? nullptr : c.take<float>((size_t)rows * in);
    o->colsum = c.take<float>(up(rows, COLSUM_ROWS) / COLSUM_ROWS * (size_t)o->piece);
    const int kw = (int)(o->rows_padded * (o->split ? TERMS : 1));
    // the last piece is shorter, and may be cut otherwise
    const int last = (int)(classes - (classes - 1) / o->piece * o->piece);
    for (int n : {(int)o->piece, last})
      partial = std::max(partial, gradient_partial_bytes(dt, rows, in, n, kw));
  }
  o->partial = (float*)c.take(partial);
  return c.bytes();
}

Operand op(const void* p, long ld, bool kc) { return Operand{p, ld, kc}; }

hipError_t launch_gradients(const Product* dx, const Product* dw, const ColumnSums* sums, const LossFinish* finish,
                            float* partial, hipStream_t st) {
  if (dx && dw) return launch_pair(*dx, *dw, sums, finish, partial, st);
  hipError_t e = sums ? launch_column_sums(*sums, st) : hipSuccess;
  if (e == hipSuccess && finish) e = launch_loss_finish(*finish, st);
  return e == hipSuccess && (dx || dw) ? launch_product(dx ? *dx : *dw, partial, st) : e;
}

}  // namespace

extern "C" {

int singa_linear_fwd_workspace_bytes(singa_dtype dtype, int rows, int in, int out, size_t* bytes) {
  if (!bytes) return SINGA_ERR_NULL;
  if (!dtype_ok(dtype)) return SINGA_ERR_UNSUPPORTED;
  const int rc = shape(rows, in, out);
  if (rc != SINGA_OK) return rc;
  FwdWs o;
  *bytes = carve_fwd(dtype, rows, in, out, nullptr, &o);
  return SINGA_OK;
}

int singa_linear_fwd(singa_dtype dtype, int rows, int in, int out, const void* x, const void* w, const float* bias,
                     singa_act act, const void* residual, void* z, void* y, void* ws, size_t ws_bytes,
                     singa_stream stream) {
  if (!dtype_ok(dtype) || act < SINGA_ACT_NONE || act > SINGA_ACT_SILU) return SINGA_ERR_UNSUPPORTED;
  int rc = shape(rows, in, out);
  if (rc != SINGA_OK) return rc;
  if (rows == 0) return SINGA_OK;
  if (!x || !w || !y) return SINGA_ERR_NULL;
  if (!aligned_to(x, 16) || !aligned_to(w, 16) || !aligned_to(y, 16) || !aligned_to(z, 16) || !aligned_to(residual, 16) ||
      !aligned_to(bias, 4))
    return SINGA_ERR_ALIGN;
  FwdWs o;
  const size_t need = carve_fwd(dtype, rows, in, out, nullptr, &o);
  rc = check_ws(ws, ws_bytes, need);
  if (rc == SINGA_OK)
    rc = check_apart({span(y, rows, out, dtype), span(z, rows, out, dtype), ws_span(ws, need)},
                     {span(x, rows, in, dtype), span(w, out, in, dtype), span(bias, 1, out, F32),
                      span(residual == y ? nullptr : residual, rows, out, dtype)});
  if (rc != SINGA_OK) return rc;
  carve_fwd(dtype, rows, in, out, ws, &o);
  hipStream_t st = (hipStream_t)stream;
  Product p;
  p.dt = dtype;
  p.M = rows;
  p.N = out;
  p.K = in;
  p.flops = 2.0 * rows * in * out;
  p.e.bias = bias;
  p.e.act = act;
  p.e.res = residual;
  p.e.z = z;
  p.e.y = y;
  if (o.skinny) {
    p.name = "skinny_kernel";
    p.a = op(x, in, true);
    p.b = op(w, in, true);
    return status(launch_skinny(p, st));
  }
  hipError_t e = hipSuccess;
  if (o.k.copy) {
    e = launch_pack2(dtype, x, o.xp, rows, w, o.wp, out, in, o.k.ld, st);
    x = o.xp;
    w = o.wp;
  }
  if (e != hipSuccess) return SINGA_ERR_HIP;
  p.name = "product_kernel<fwd>";
  p.a = op(x, o.k.ld, true);
  p.b = op(w, o.k.ld, true);
  return status(launch_product(p, o.partial, st));
}

int singa_linear_bwd_workspace_bytes(singa_dtype dtype, int rows, int in, int out, singa_act act, singa_dtype dw_dtype,
                                     size_t* bytes) {
  if (!bytes) return SINGA_ERR_NULL;
  if (!dtype_ok(dtype) || !dtype_ok(dw_dtype) || act < SINGA_ACT_NONE || act > SINGA_ACT_SILU) return SINGA_ERR_UNSUPPORTED;
  if (dw_dtype == SINGA_BF16 && dtype != SINGA_BF16) return SINGA_ERR_UNSUPPORTED;
  const int rc = shape(rows, in, out);
  if (rc != SINGA_OK) return rc;
  BwdWs o;
  *bytes = carve_bwd(dtype, rows, in, out, act, dw_dtype, nullptr, &o);
  return SINGA_OK;
}

int singa_linear_bwd(singa_dtype dtype, int rows, int in, int out, const void* x, const void* w, const void* z, singa_act act,
                     const void* dy, const void* dx_residual, void* dx, void* dw, singa_dtype dw_dtype, float* db,
                     int accumulate, void* ws, size_t ws_bytes, singa_stream stream) {
  size_t need = 0;
  int rc = singa_linear_bwd_workspace_bytes(dtype, rows, in, out, act, dw_dtype, &need);
  if (rc != SINGA_OK) return rc;
  if (dw && dw_dtype == SINGA_BF16 && accumulate) return SINGA_ERR_UNSUPPORTED;
  if (rows && !dx && !dw && !db) return SINGA_ERR_NULL;  // (a dx of no rows has no address)
  if (rows && (!dy || (dw && !x) || (dx && !w) || (act != SINGA_ACT_NONE && !z))) return SINGA_ERR_NULL;
  if (!aligned_to(x, 16) || !aligned_to(w, 16) || !aligned_to(z, 16) || !aligned_to(dy, 16) || !aligned_to(dx_residual, 16) ||
      !aligned_to(dx, 16) || !aligned_to(dw, 16) || !aligned_to(db, 4))
    return SINGA_ERR_ALIGN;
  rc = check_ws(ws, ws_bytes, need);
  if (rc != SINGA_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
  hipError_t e = hipSuccess;
  if (rows == 0) {
    if (accumulate) return SINGA_OK;
    if (dw) e = launch_zero(dw, (size_t)out * in * dt_size(dw_dtype), st);
    if (e == hipSuccess && db) e = launch_zero(db, (size_t)out * 4, st);
    return status(e);
  }
  rc = check_apart({span(dx, rows, in, dtype), span(dw, out, in, dw_dtype), span(db, 1, out, F32), ws_span(ws, need)},
                   {span(dw ? x : nullptr, rows, in, dtype), span(dx ? w : nullptr, out, in, dtype), span(dy, rows, out, dtype),
                    span(act == SINGA_ACT_NONE ? nullptr : z, rows, out, dtype),
                    span(!dx || dx_residual == dx ? nullptr : dx_residual, rows, in, dtype)});
  if (rc != SINGA_OK) return rc;
  BwdWs o;
  carve_bwd(dtype, rows, in, out, act, dw_dtype, ws, &o);
  const bool split = o.split && dw;
  // few rows of a dy that goes into the products as it is: db straight from it
  const bool direct = !o.own_dz && rows <= FINISH_ROWS;
  if (o.own_dz || (db && !direct))
    e = launch_dact(dtype, act, dy, z, o.own_dz ? o.dz : nullptr, split ? o.more : nullptr, db ? o.colsum : nullptr, rows,
                    o.rows_padded, out, o.ldz, st);
  const ColumnSums sums = direct ? ColumnSums{dy, dtype, rows, out, db, accumulate, nullptr}
                                 : ColumnSums{o.colsum, F32, o.groups, out, db, accumulate, nullptr};
  const void* dz = o.own_dz ? o.dz : dy;
  if (o.k.copy && (dx || dw) && e == hipSuccess) {
    e = launch_pack2(dtype, x, o.xp, dw ? rows : 0, w, o.wp, dx ? out : 0, in, o.k.ld, st);
    x = o.xp;
    w = o.wp;
  }
  Product p, q;
  p.dt = q.dt = dtype;
  p.flops = q.flops = 2.0 * rows * in * out;
  if (dx) {
    p.name = "product_kernel<bwd_data>";
    p.M = rows;
    p.N = in;
    p.K = out;
    p.a = op(dz, o.ldz, true);
    p.b = op(w, o.k.ld, false);
    p.e.res = dx_residual;
    p.e.y = dx;
  }
  if (dw) {
    q.name = "product_kernel<bwd_weights>";
    q.M = out;
    q.N = in;
    q.K = split ? (int)(TERMS * o.rows_padded) : rows;
    q.wrap = split ? (int)o.rows_padded : 0;
    q.kb = rows;
    q.a = op(dz, o.ldz, false);
    q.b = op(x, o.k.ld, false);
    q.e.y = dw;
    q.e.out_f32 = dw_dtype == SINGA_F32;
    q.e.add = accumulate != 0;
  }
  if (e == hipSuccess) e = launch_gradients(dx ? &p : nullptr, dw ? &q : nullptr, db ? &sums : nullptr, nullptr, o.partial, st);
  return status(e);
}

int singa_linear_softmax_ce_workspace_bytes(singa_dtype dtype, int rows, int in, int classes, int gradients,
                                            singa_dtype dw_dtype, size_t* bytes) {
  if (!bytes) return SINGA_ERR_NULL;
  if (!dtype_ok(dtype) || !dtype_ok(dw_dtype)) return SINGA_ERR_UNSUPPORTED;
  if (dw_dtype == SINGA_BF16 && dtype != SINGA_BF16) return SINGA_ERR_UNSUPPORTED;
  const int rc = shape(rows, in, classes);
  if (rc != SINGA_OK) return rc;
  LossWs o;
  *bytes = carve_loss(dtype, rows, in, classes, gradients != 0, dw_dtype, nullptr, &o);
  return SINGA_OK;
}

int singa_linear_softmax_ce(singa_dtype dtype, int rows, int in, int classes, const void* x, const void* w, const float* bias,
                            const int32_t* labels, float scale, float* loss, void* dx, void* dw, singa_dtype dw_dtype,
                            float* db, int accumulate, void* ws, size_t ws_bytes, singa_stream stream) {
  const bool grad = dx || dw || db;
  size_t need = 0;
  int rc = singa_linear_softmax_ce_workspace_bytes(dtype, rows, in, classes, grad, dw_dtype, &need);
  if (rc != SINGA_OK) return rc;
  if (dw && dw_dtype == SINGA_BF16 && accumulate) return SINGA_ERR_UNSUPPORTED;
  if (!loss || !w || (rows && (!x || !labels))) return SINGA_ERR_NULL;
  if (!aligned_to(x, 16) || !aligned_to(w, 16) || !aligned_to(dx, 16) || !aligned_to(dw, 16) || !aligned_to(bias, 4) ||
      !aligned_to(labels, 4) || !aligned_to(loss, 4) || !aligned_to(db, 4))
    return SINGA_ERR_ALIGN;
  rc = check_ws(ws, ws_bytes, need);
  if (rc != SINGA_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
  hipError_t e = hipSuccess;
  if (rows == 0) {
    e = launch_zero(loss, 4, st);
    if (e == hipSuccess && dw && !accumulate) e = launch_zero(dw, (size_t)classes * in * dt_size(dw_dtype), st);
    if (e == hipSuccess && db && !accumulate) e = launch_zero(db, (size_t)classes * 4, st);
    return status(e);
  }
  rc = check_apart({{loss, (size_t)(rows + 1L) * 4}, span(dx, rows, in, dtype), span(dw, classes, in, dw_dtype),
                    span(db, 1, classes, F32), ws_span(ws, need)},
                   {span(x, rows, in, dtype), span(w, classes, in, dtype), span(bias, 1, classes, F32),
                    span(labels, rows, 1, F32)});
  if (rc != SINGA_OK) return rc;
  LossWs o;
  carve_loss(dtype, rows, in, classes, grad, dw_dtype, ws, &o);
  const void *xt = x, *wt = w;  // as the tiles take them
  if (o.wp) {
    e = launch_pack2(dtype, x, o.xp, rows, w, o.wp, classes, in, o.k.ld, st);
    wt = o.wp;
    xt = o.xp;
  }
  Product p;
  p.dt = dtype;
  p.M = rows;
  p.N = classes;
  p.K = in;
  p.flops = 2.0 * rows * in * classes;
  p.e.bias = bias;
  p.e.labels = labels;
  p.e.classes = classes;
  if (o.skinny) {
    p.a = op(x, in, true);
    p.b = op(w, in, true);
  } else {
    p.a = op(xt, o.k.ld, true);
    p.b = op(wt, o.k.ld, true);
  }
  const bool split = o.split && dw;
  void* more = split ? o.more : nullptr;
  const long groups = up(rows, COLSUM_ROWS) / COLSUM_ROWS;
  // few rows of kept logits: the mean and db with the gradients' launch
  const bool finish = o.keep && rows <= FINISH_ROWS;
  const LossFinish fin{labels, classes, rows, loss, scale, o.logits, o.ldl, db, accumulate};
  if (o.keep) {
    // the logits, then their rows
    Product q = p;
    q.e = Epilogue{};
    q.e.y = o.logits;  // few rows' kernel
    q.e.ldy = o.ldl;
    q.e.out_f32 = 1;
    q.raw = true;
    if (e == hipSuccess) {
      q.name = o.skinny ? "skinny_kernel" : "product_kernel<logits>";
      e = o.skinny ? launch_skinny(q, st) : launch_product(q, o.logits, st);
    }
    LossRows r{};
    r.z = o.logits;
    r.ldz = o.ldl;
    r.splits = o.splits;
    r.bias = bias;
    r.labels = labels;
    r.rows = rows;
    r.rows_padded = o.rows_padded;
    r.classes = classes;
    r.loss = loss;
    r.stats = o.stats;
    r.unit = grad && finish ? o.unit : nullptr;
    r.scale = scale;
    if (!grad) {
      r.rows_padded = rows;
    } else {
      r.dz = o.dz;
      r.more = more;
      r.ldd = o.ldd;
      r.keep_dz = db != nullptr;
    }
    if (dw) {
      r.x = x;
      r.xc = o.xc;
      r.in = in;
      r.ldx = o.k.ld;
    }
    if (e == hipSuccess) e = launch_loss_rows(dtype, r, st);
    if (e == hipSuccess && finish && !grad) e = launch_loss_finish(fin, st);
  } else {
    p.epi = EPI_LSE;
    p.e.stats = o.stats;
    p.e.nstat = o.nstat;
    p.e.zlab = o.zlab;
    if (e == hipSuccess) {
      p.name = o.skinny ? "skinny_kernel" : "product_kernel<lse>";
      e = o.skinny ? launch_skinny(p, st) : launch_product(p, nullptr, st);
    }
    if (!grad && lse_finish_pays(rows, o.nstat))
      return status(e == hipSuccess ? launch_lse_finish(o.stats, o.nstat, o.zlab, labels, classes, rows, loss, st) : e);
    if (e == hipSuccess) e = launch_lse(o.stats, o.nstat, o.zlab, labels, classes, rows, o.lse, loss, st);
  }
  if (e == hipSuccess && !finish) e = launch_loss_mean(labels, classes, rows, loss, grad ? o.unit : nullptr, scale, st);
  if (!grad || e != hipSuccess) return status(e);

  // x without its padding rows, for dw: a zero gradient times what they hold
  // need not be zero
  if (dw && !o.keep) e = launch_pack(dtype, x, o.xc, rows, in, o.k.ld, labels, classes, st);
  const long es = (long)dt_size(dtype);
  for (long c0 = 0; c0 < classes && e == hipSuccess; c0 += o.piece) {
    const int n = (int)std::min(o.piece, classes - c0);
    const char* wc = (const char*)wt + c0 * o.k.ld * es;
    if (!o.keep) {
      Product q = p;
      q.name = "product_kernel<dlogits>";
      q.epi = EPI_DLOGITS;
      q.N = n;
      q.flops = 2.0 * rows * in * n;
      q.a = op(xt, o.k.ld, true);
      q.b = op(wc, o.k.ld, true);
      q.e.bias = bias ? bias + c0 : nullptr;
      q.e.col0 = (int)c0;
      q.e.lse = o.lse;
      q.e.y = o.dz;
      q.e.ldy = o.ldd;
      q.e.more = (bf16_t*)more;
      q.e.rows_padded = (int)o.rows_padded;
      q.e.colsum = db ? o.colsum : nullptr;
      e = launch_product(q, nullptr, st);
    } else if (db && !finish) {
      e = launch_colsum_rows(o.logits, o.ldl, o.colsum, rows, classes, labels, classes, st);
    }
    const ColumnSums sums{o.colsum, F32, groups, n, db ? db + c0 : nullptr, accumulate, o.unit};
    Product q, v;
    if (dx) {
      q.name = "product_kernel<bwd_data>";
      q.dt = dtype;
      q.flops = 2.0 * rows * in * n;
      q.M = rows;
      q.N = in;
      q.K = n;
      q.a = op(o.dz, o.ldd, true);
      q.b = op(wc, o.k.ld, false);
      q.e.alpha = o.unit;
      q.e.y = o.one ? dx : (void*)o.dxf;
      q.e.out_f32 = !o.one;
      q.e.add = !o.one && c0 > 0;
      if (o.one) {
        q.e.labels = labels;
        q.e.classes = classes;
      }
    }
    if (dw) {
      v.name = "product_kernel<bwd_weights>";
      v.dt = dtype;
      v.flops = 2.0 * rows * in * n;
      v.M = n;
      v.N = in;
      v.K = split ? (int)(TERMS * o.rows_padded) : rows;
      v.wrap = split ? (int)o.rows_padded : 0;
      v.kb = rows;
      v.a = op(o.dz, o.ldd, false);
      v.b = op(o.xc, o.k.ld, false);
      v.e.alpha = o.unit;
      v.e.y = (char*)dw + c0 * in * (long)dt_size(dw_dtype);
      v.e.out_f32 = dw_dtype == SINGA_F32;
      v.e.add = accumulate != 0;
    }
    if (e == hipSuccess)
      e = launch_gradients(dx ? &q : nullptr, dw ? &v : nullptr, db && !finish ? &sums : nullptr, finish ? &fin : nullptr,
                           o.partial, st);
  }
  if (e == hipSuccess && dx && !o.one) e = launch_round_rows(dtype, o.dxf, dx, rows, in, labels, classes, st);
  return status(e);
}

size_t singa_grad_norm_workspace_bytes(int count) { return count < 0 ? 0 : norm_slots(count) * sizeof(double); }

// Clipping writes one tensor while it reads another: outputs may share memory
// with nothing but the gradient they stand for (a gradient listed twice would
// be scaled once or twice, as the workgroups happen to run).
static int clip_apart(int count, const int* dtypes, const void* const* grads, void* const* outs, const size_t* sizes) {
  struct Part {
    uintptr_t lo, hi;
    bool written;
  };
  const std::unique_ptr<Part[]> parts(new (std::nothrow) Part[2 * (size_t)count]);
  if (!parts) return SINGA_ERR_HIP;
  Part* end = parts.get();
  for (int i = 0; i < count; ++i) {
    if (!sizes[i]) continue;
    const size_t bytes = sizes[i] * dt_size(dtypes[i]);
    *end++ = {(uintptr_t)outs[i], (uintptr_t)outs[i] + bytes, true};
    if (grads[i] != outs[i]) *end++ = {(uintptr_t)grads[i], (uintptr_t)grads[i] + bytes, false};
  }
  std::sort(parts.get(), end, [](const Part& a, const Part& b) { return a.lo < b.lo; });
  uintptr_t read = 0, written = 0;  // the ends of what came before
  for (const Part* p = parts.get(); p < end; ++p) {
    if (p->lo < written || (p->written && p->lo < read)) return SINGA_ERR_UNSUPPORTED;
    (p->written ? written : read) = std::max(p->written ? written : read, p->hi);
  }
  return SINGA_OK;
}

static int grad_norm(int count, const int* dtypes, const void* const* grads, void* const* outs, bool clip, const size_t* sizes,
                     float max_norm, float* stat, void* ws, size_t ws_bytes, singa_stream stream) {
  if (count < 0) return SINGA_ERR_SHAPE;
  if (!(max_norm >= 0.f)) return SINGA_ERR_UNSUPPORTED;
  if (!stat || (count && (!dtypes || !grads || !sizes || (clip && !outs)))) return SINGA_ERR_NULL;
  for (int i = 0; i < count; ++i) {
    if (!dtype_ok(dtypes[i])) return SINGA_ERR_UNSUPPORTED;
    if (!sizes[i]) continue;
    if (sizes[i] > (size_t)1 << 40) return SINGA_ERR_SHAPE;
    if (!grads[i] || (clip && !outs[i])) return SINGA_ERR_NULL;
    if (!aligned_to(grads[i], dt_size(dtypes[i])) || (clip && !aligned_to(outs[i], dt_size(dtypes[i])))) return SINGA_ERR_ALIGN;
  }
  if (!aligned_to(stat, 4)) return SINGA_ERR_ALIGN;
  const size_t need = singa_grad_norm_workspace_bytes(count);
  int rc = check_ws(ws, ws_bytes, need);
  // the gradients that are only read may share memory with each other
  const Span own[] = {{stat, 2 * sizeof(float)}, ws_span(ws, need)};
  if (rc == SINGA_OK && !apart(own[0], own[1])) rc = SINGA_ERR_UNSUPPORTED;
  for (int i = 0; i < count && rc == SINGA_OK; ++i) {
    const Span g{sizes[i] ? grads[i] : nullptr, sizes[i] * dt_size(dtypes[i])}, o{clip && sizes[i] ? outs[i] : nullptr, g.bytes};
    for (const Span& w : own)
      if (!apart(w, g) || !apart(w, o)) rc = SINGA_ERR_UNSUPPORTED;
  }
  if (rc == SINGA_OK && clip && count) rc = clip_apart(count, dtypes, grads, outs, sizes);
  if (rc != SINGA_OK) return rc;
  return status(launch_grad_norm(count, dtypes, grads, clip ? outs : nullptr, sizes, max_norm, stat, (double*)ws,
                                 (hipStream_t)stream));
}

int singa_grad_norm(int count, const int* dtypes, const void* const* grads, const size_t* sizes, float max_norm, float* stat,
                    void* ws, size_t ws_bytes, singa_stream stream) {
  return grad_norm(count, dtypes, grads, nullptr, false, sizes, max_norm, stat, ws, ws_bytes, stream);
}

int singa_grad_clip(int count, const int* dtypes, const void* const* grads, void* const* outs, const size_t* sizes,
                    float max_norm, float* stat, void* ws, size_t ws_bytes, singa_stream stream) {
  return grad_norm(count, dtypes, grads, outs, true, sizes, max_norm, stat, ws, ws_bytes, stream);
}

// An update's own streams and the factor that every thread reads.
static int update_apart(size_t n, const float* w, const float* g, const float* v, const uint16_t* w_bf16, const float* scale) {
  return check_apart({Span{w, n * 4}, Span{v, n * 4}, Span{w_bf16, n * 2}}, {Span{g, n * 4}, Span{scale, 4}});
}

int singa_sgd_momentum_update_scaled(size_t n, float* w, const float* g, float* v, uint16_t* w_bf16, float lr, float momentum,
                                     float weight_decay, const float* grad_scale, singa_stream stream) {
  if (n == 0) return SINGA_OK;
  if (!w || !g || !v || !grad_scale) return SINGA_ERR_NULL;
  if (!aligned_to(w, 16) || !aligned_to(g, 16) || !aligned_to(v, 16) || !aligned_to(w_bf16, 16) || !aligned_to(grad_scale, 4))
    return SINGA_ERR_ALIGN;
  if (update_apart(n, w, g, v, w_bf16, grad_scale) != SINGA_OK) return SINGA_ERR_UNSUPPORTED;
  return status(launch_sgd_scaled(n, w, g, v, w_bf16, lr, momentum, weight_decay, grad_scale, (hipStream_t)stream));
}

int singa_adagrad_update_scaled(size_t n, float* w, const float* g, float* h, uint16_t* w_bf16, float lr, float delta,
                                float weight_decay, const float* grad_scale, singa_stream stream) {
  if (n == 0) return SINGA_OK;
  if (!w || !g || !h || !grad_scale) return SINGA_ERR_NULL;
  if (!aligned_to(w, 16) || !aligned_to(g, 16) || !aligned_to(h, 16) || !aligned_to(w_bf16, 16) || !aligned_to(grad_scale, 4))
    return SINGA_ERR_ALIGN;
  if (!(delta > 0.f) || !(lr >= 0.f) || update_apart(n, w, g, h, w_bf16, grad_scale) != SINGA_OK) return SINGA_ERR_UNSUPPORTED;
  return status(launch_adagrad_scaled(n, w, g, h, w_bf16, lr, delta, weight_decay, grad_scale, (hipStream_t)stream));
}

}  // extern "C"
