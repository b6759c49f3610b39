// dense_gemm.h -- the tile kernel of the dense products (see dense.h).
//
// A workgroup computes a BM x BN tile; the K range goes through LDS in tiles
// of 128 bytes (64 bf16 or 32 fp32 values of k), written there straight from
// memory (buffer loads to LDS), two stages.  An operand is staged the way
// it is stored:
//   K contiguous:    BM rows of 128 bytes; a lane's fragment (8 bf16 or 4 fp32
//                    of one row) is one 16-byte read.  16-byte chunk c of row
//                    r lies in slot c ^ (r / 2 % 8), so that 16 rows read at
//                    the same k touch 16 different 16-byte groups of banks.
//   rows contiguous: 64 (32) rows of k; bf16 fragments come from transposing
//                    LDS reads (four k of 16 rows each), fp32 ones from four
//                    4-byte reads.  Chunk c of k row d lies in slot
//                    c ^ 4 (d % 4) (bf16) or c ^ 8 (d / 4 % 2) (fp32): the
//                    rows that one read touches lie in different banks.
// Both operands take their k in the same order, so either type's fragments
// feed the matrix instruction as they come: v_mfma_f32_32x32x16_bf16 once or
// v_mfma_f32_32x32x2_f32 four times per 16 bytes.  Sums are fp32.
#pragma once

#include "conv_common.h"
#include "dense.h"

namespace singa {

namespace {

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

struct GemmArgs {
  const char *a, *b;
  long lda, ldb;            // bytes
  long enda, endb;          // bytes of the whole operand
  int M, N;
  int kca, kcb;             // 16-byte chunks of K (K contiguous operands)
  int kt_all, kt_split, splits, wrap;  // K-tiles: all, per split, splits, where B starts again (0: never)
  int tiles_m, tiles_n;
  float* partial;           // [splits][M][ldp] when splits > 1
  long ldp;
  int raw;                  // the sums as they are go to `partial`
  int vec;                  // outputs take 16-byte vectors
  Epilogue e;
};

__device__ __forceinline__ v4i16 lds_tr16(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) v4i16*)(__attribute__((address_space(3))) char*)p);
}

// exp in the hardware's base-2 form: x log2(e) is rounded once, so the result
// is off by at most |x| 2^-24 relative besides the instruction's own ulp.  A
// softmax's x is not above 0, and what matters of it lies at small |x|; the
// activations in bf16, where x may be up to 88 before it overflows to the right
// limit, lose 2^-17 of a value that is rounded to 2^-8.
__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }

// A row of a softmax, from the maximum m of its logits and the sum s of their
// exponentials relative to it.  m and the logarithm of s stay apart: their
// rounded sum would be off by half an ulp of m, which an offset of all logits
// makes as large as it likes (at 65536 a loss of 0.0616 came out as 0.0625).
__device__ __forceinline__ float2 row_lse(float m, float s) { return make_float2(m, log2f(s)); }
__device__ __forceinline__ float row_loss(float m, float s, float zlab) { return (m - zlab) + logf(s); }
// The probability of logit z: 2^((z - m) log2(e) - log2(s)).
__device__ __forceinline__ float row_prob(float z, float2 lse) {
  return __builtin_amdgcn_exp2f(fmaf(z - lse.x, 1.44269504088896341f, -lse.y));
}

// erfc(x) exp(x^2) for x >= 0: t q(t) with t = 1 / (1 + 0.4375 x) and a
// polynomial q fitted for the smallest relative error over x <= 14 (reweighted
// least squares), 1.7e-7, 4.5e-7 as evaluated here: gelu's values far below
// zero, where erfc is small, are right as well.
__device__ __forceinline__ float erfc_poly(float x) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.4375f, x, 1.f));
  const float a = fmaf(t, fmaf(t, fmaf(t, 0.0718273446f, -0.28582573f), 0.317387909f), -0.0351383798f);
  return t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, a, 0.222752094f), 0.214494616f), 0.247705251f), 0.246796981f);
}

// act(z).  bf16 results are rounded to 2^-8: the hardware's exponential and
// reciprocal and the polynomial do; fp32 results take the library's functions.
template <typename T> __device__ __forceinline__ float act_f(float z, int act) {
  constexpr bool FAST = sizeof(T) == 2;
  if (act == ACT_RELU) return z > 0.f ? z : (z != z ? z : 0.f);
  if (act == ACT_GELU) {
    if constexpr (FAST) {
      const float u = fabsf(z) * 0.70710678118654752f;
      const float h = 0.5f * erfc_poly(u) * exp_fast(-u * u);
      return z * (z < 0.f ? h : 1.f - h);
    }
    return 0.5f * z * erfcf(-z * 0.70710678118654752f);
  }
  if (act == ACT_SILU) {
    if constexpr (FAST) return z * __builtin_amdgcn_rcpf(1.f + exp_fast(-z));
    return z / (1.f + expf(-z));
  }
  return z;
}

// act'(z): dz = dy act'(z)
template <typename T> __device__ __forceinline__ float act_slope(float z, int act) {
  if (act == ACT_RELU) return z > 0.f ? 1.f : 0.f;
  constexpr bool FAST = sizeof(T) == 2;  // 5e-7 off at most
  if (act == ACT_GELU) {
    if constexpr (FAST) {  // one exponential serves both terms
      const float u = fabsf(z) * 0.70710678118654752f, e = exp_fast(-u * u), h = 0.5f * erfc_poly(u) * e;
      return fmaf(z * 0.39894228040143268f, e, z < 0.f ? h : 1.f - h);
    }
    return fmaf(z * 0.39894228040143268f, expf(-0.5f * z * z), 0.5f * erfcf(-z * 0.70710678118654752f));
  }
  if (act == ACT_SILU) {
    const float s = FAST ? __builtin_amdgcn_rcpf(1.f + exp_fast(-z)) : 1.f / (1.f + expf(-z));
    return s * fmaf(z, 1.f - s, 1.f);
  }
  return 1.f;
}

// ------------------------------------------------------------- epilogues
template <typename T> __device__ __forceinline__ void load8(const T* p, float (&v)[8]);
template <> __device__ __forceinline__ void load8<float>(const float* p, float (&v)[8]) {
  const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = a[j], v[4 + j] = b[j];
}
template <> __device__ __forceinline__ void load8<bf16_t>(const bf16_t* p, float (&v)[8]) {
  const uint4 u = *(const uint4*)p;
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = __uint_as_float(w[j] << 16);
    v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
  }
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&v)[8]);
template <> __device__ __forceinline__ void store8<float>(float* p, const float (&v)[8]) {
  *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
  *(f32x4*)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}
template <> __device__ __forceinline__ void store8<bf16_t>(bf16_t* p, const float (&v)[8]) {
  *(u32x4_t*)p = u32x4_t{f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]),
                         f32x2_to_bf16x2(v[6], v[7])};
}

// The value of lane l ^ d for d = 1, 2; for d = 4 that of the lane mirrored in
// its group of 8, which holds the same once groups of 4 agree.  Data-parallel
// moves, no LDS round trip.
__device__ __forceinline__ float lane_xor(float v, int d) {
  const int x = __float_as_int(v);
  return __int_as_float(d == 1   ? __builtin_amdgcn_update_dpp(0, x, 0xb1, 0xf, 0xf, true)   // quad_perm [1,0,3,2]
                        : d == 2 ? __builtin_amdgcn_update_dpp(0, x, 0x4e, 0xf, 0xf, true)   // quad_perm [2,3,0,1]
                                 : __builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, true));  // row_half_mirror
}

// v at y + o and, with more, its further terms, `step` elements apart.
template <typename T>
__device__ __forceinline__ void store_terms(T* y, bf16_t* more, size_t o, size_t step, float (&v)[8]) {
  store8<T>(y + o, v);
  if constexpr (sizeof(T) == 2) {
    if (more) {
#pragma unroll
      for (int t = 0; t < TERMS - 1; ++t) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] -= bf16_to_f32(f32_to_bf16(v[j]));
        store8<bf16_t>(more + t * step + o, v);
      }
    }
  }
}

__device__ __forceinline__ bool label_ok(int lab, int classes) { return lab >= 0 && lab < classes; }

// What EPI_OUT adds to or multiplies with a lane's 8 columns in every row.
struct Columns {
  float alpha, bias[8];
};
__device__ __forceinline__ Columns columns_of(const Epilogue& e, int N, int col, int colb) {
  Columns c;
  c.alpha = e.alpha ? e.alpha[0] : 1.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int k = j < 4 ? col + j : colb + j - 4;
    c.bias[j] = e.bias && k < N ? e.bias[k] : 0.f;
  }
  return c;
}

// What EPI_OUT adds to 8 values of a row (the residual, or what y holds): two
// 16-byte vectors of fp32, or one of bf16.
struct Extra {
  uint4 a, b;
};
template <typename T>
__device__ __forceinline__ Extra load_extra(const Epilogue& e, int M, int N, int row, int col, int colb) {
  // every lane reads (element 0 stands in for what lies outside), so that no
  // load sits in a branch that the next one waits for
  Extra x;
  const bool in = row < M && col < N, inb = row < M && colb < N;
  if (e.add) {
    const float* p = (const float*)e.y;
    x.a = *(const uint4*)(p + (in ? (size_t)row * e.ldy + col : 0));
    x.b = *(const uint4*)(p + (inb ? (size_t)row * e.ldy + colb : 0));
  } else {
    const T* p = (const T*)e.res;
    x.a = *(const uint4*)(p + (in ? (size_t)row * N + col : 0));
    x.b = sizeof(T) == 4 ? *(const uint4*)(p + (inb ? (size_t)row * N + colb : 0)) : x.a;
  }
  return x;
}
template <typename T> __device__ __forceinline__ void add_extra(bool f32, const Extra& x, float (&v)[8]) {
  const uint32_t a[4] = {x.a.x, x.a.y, x.a.z, x.a.w}, b[4] = {x.b.x, x.b.y, x.b.z, x.b.w};
  if (sizeof(T) == 4 || f32) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] += __uint_as_float(a[j]);
      v[4 + j] += __uint_as_float(b[j]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] += __uint_as_float(a[j] << 16);
      v[2 * j + 1] += __uint_as_float(a[j] & 0xffff0000u);
    }
  }
}

// The activation of n values: one branch for all, so that their chains of
// dependent instructions overlap.
template <typename T, int n> __device__ __forceinline__ void act_all(float (&v)[n], int act) {
  if (act == ACT_RELU) {
#pragma unroll
    for (int j = 0; j < n; ++j) v[j] = act_f<T>(v[j], ACT_RELU);
  } else if (act == ACT_GELU) {
#pragma unroll
    for (int j = 0; j < n; ++j) v[j] = act_f<T>(v[j], ACT_GELU);
  } else if (act == ACT_SILU) {
#pragma unroll
    for (int j = 0; j < n; ++j) v[j] = act_f<T>(v[j], ACT_SILU);
  }
}

// EPI_OUT on 8 columns of R rows, in 16-byte vectors (N % 8 == 0 and every
// tensor starts at a 16-byte boundary).  x: what is added (e.res or e.add);
// live: false where a label takes the row out; put_z, put_y: store row u;
// before_y: what goes between the last use of x and the stores.
template <typename T, int R, typename PutZ, typename PutY, typename Before>
__device__ __forceinline__ void epi_out(const Epilogue& e, float (&v)[R][8], const Columns& c, const Extra (&x)[R],
                                        const bool (&live)[R], PutZ put_z, PutY put_y, Before before_y) {
#pragma unroll
  for (int u = 0; u < R; ++u)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[u][j] = fmaf(v[u][j], c.alpha, c.bias[j]);
  if (e.z) {
#pragma unroll
    for (int u = 0; u < R; ++u) put_z(u, v[u]);
  }
  if (e.act) {
#pragma unroll
    for (int u = 0; u < R; ++u) act_all<T, 8>(v[u], e.act);
  }
  if (e.labels) {
#pragma unroll
    for (int u = 0; u < R; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[u][j] = live[u] ? v[u][j] : 0.f;
  }
  if (e.res || e.add) {
#pragma unroll
    for (int u = 0; u < R; ++u) add_extra<T>(e.add, x[u], v[u]);
  }
  before_y();
#pragma unroll
  for (int u = 0; u < R; ++u) put_y(u, v[u]);
}

// Four fp32 values, or eight as bf16, at byte offset o of a buffer (past its
// end: not stored, and no branch that the stores around it would have to be
// counted across).  NT: non-temporal, for outputs that this launch does not
// read again (8192^3: 819 -> 810 us).
template <bool NT> __device__ __forceinline__ void buf_store4(__amdgpu_buffer_rsrc_t r, uint32_t o, const float* v) {
  const u32x4_t p = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  __builtin_amdgcn_raw_buffer_store_b128(p, r, (int)o, 0, NT ? 2 : 0);
}
template <bool NT> __device__ __forceinline__ void buf_store8h(__amdgpu_buffer_rsrc_t r, uint32_t o, const float (&v)[8]) {
  const u32x4_t p = {f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]),
                     f32x2_to_bf16x2(v[6], v[7])};
  __builtin_amdgcn_raw_buffer_store_b128(p, r, (int)o, 0, NT ? 2 : 0);
}

// The same, element by element, for any N.
template <typename T>
__device__ __forceinline__ void epi_out_any(const Epilogue& e, int N, int row, int col, int colb, const float (&v)[8],
                                            const Columns& c, bool live) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int k = j < 4 ? col + j : colb + j - 4;
    if (k >= N) continue;
    const size_t o = (size_t)row * N + k, oy = (size_t)row * e.ldy + k;
    float y = fmaf(v[j], c.alpha, c.bias[j]);
    if (e.z) store_out<T>((T*)e.z + o, y);
    if (e.act) y = act_f<T>(y, e.act);
    if (!live) y = 0.f;
    if (e.res) y += elem_f(((const T*)e.res)[o]);
    if (e.add) y += ((const float*)e.y)[oy];
    if (e.out_f32)
      ((float*)e.y)[oy] = y;
    else
      store_out<T>((T*)e.y + oy, y);
  }
}

template <int V> struct Const { static constexpr int value = V; };

template <typename T> struct TypeInfo;
template <> struct TypeInfo<bf16_t> {
  static constexpr int VEC = 8, BK = 64;
};
template <> struct TypeInfo<float> {
  static constexpr int VEC = 4, BK = 32;
};

template <typename T> struct Chunk;
template <> struct Chunk<bf16_t> { typedef bf16x8 type; };
template <> struct Chunk<float> { typedef f32x4 type; };

__device__ __forceinline__ void mma32(const bf16x8& a, const bf16x8& b, f32x16& c) {
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ void mma32(const f32x4& a, const f32x4& b, f32x16& c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
}

// One operand's tile: R rows of the product by one K-tile, in LDS, with NW
// waves loading it.  W0: the first of this wave's rows.
template <typename T, bool KC, int R, int NW> struct Tile {
  static constexpr int ES = (int)sizeof(T), VEC = TypeInfo<T>::VEC, BK = TypeInfo<T>::BK;
  static constexpr int BYTES = R * 128;
  static constexpr int NI = BYTES / 1024 / NW;  // load instructions per wave and K-tile
  static_assert(BYTES % (1024 * NW) == 0, "whole instructions");
  static constexpr int RB = R * ES;             // rows contiguous: bytes of a k row
  static constexpr int CPR = RB / 16;

  uint32_t off[NI];  // within the tile's rsrc; OOB: nothing to read

  // K contiguous: the chunk of the K-tile that instruction i of this lane loads
  __device__ __forceinline__ static int chunk(int wave, int lane, int i) {
    return (lane & 7) ^ ((((wave * NI + i) * 8 + (lane >> 3)) >> 1) & 7);
  }
  __device__ __forceinline__ void init(int wave, int lane, long ld, int r0, int rows) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int idx = wave * NI + i;
      if constexpr (KC) {
        const int r = idx * 8 + (lane >> 3);
        off[i] = r0 + r < rows ? (uint32_t)(r * ld + chunk(wave, lane, i) * 16) : OOB;
      } else {
        constexpr int RPI = 1024 / RB;
        const int d = idx * RPI + lane / CPR;
        const int c = (lane % CPR) ^ (ES == 2 ? 4 * (d & 3) : 8 * ((d >> 2) & 1));
        off[i] = r0 + c * VEC < (rows + VEC - 1) / VEC * VEC ? (uint32_t)(d * ld + c * 16) : OOB;
      }
    }
  }
  // the last K-tile holds only kleft chunks of K
  __device__ __forceinline__ void mask(int wave, int lane, int kleft) {
    if constexpr (KC) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (chunk(wave, lane, i) >= kleft) off[i] = OOB;
    }
  }
  // instruction i of this wave; lds: the LDS address of the wave's part
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rs, uint32_t lds, int i) const {
    asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds + i * 1024), "v"(off[i]), "s"(rs)
                 : "memory");
  }
};

// Fragment reads of one operand for a wave: F blocks of 32 rows from w0.
template <typename T, bool KC, int R, int F> struct Frags {
  static constexpr int ES = (int)sizeof(T);
  static constexpr int RB = R * ES;
  int addr[KC ? 4 : F];
  __device__ __forceinline__ void init(int lane, int w0) {
    const int li = lane & 31, lh = lane >> 5;
    if constexpr (KC) {
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) addr[ks] = (w0 + li) * 128 + (((2 * ks + lh) ^ ((li >> 1) & 7)) << 4);
    } else if constexpr (ES == 2) {
      const int row = 8 * lh + ((lane & 15) >> 2), rr = row & 3;
      const int low = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), odd = 8 * (lane & 1);
#pragma unroll
      for (int b = 0; b < F; ++b) addr[b] = row * RB + ((4 * ((w0 / 32 + b) ^ rr) + low) << 4) + odd;
    } else {
#pragma unroll
      for (int b = 0; b < F; ++b) {
        const int col = w0 + b * 32 + li;
        addr[b] = 4 * lh * RB + (((col >> 2) ^ (8 * lh)) << 4) + (col & 3) * 4;
      }
    }
  }
  __device__ __forceinline__ typename Chunk<T>::type read(const char* s, int b, int ks) const {
    if constexpr (KC) {
      return *(const typename Chunk<T>::type*)(s + addr[ks] + b * 32 * 128);
    } else if constexpr (ES == 2) {
      const v4i16 lo = lds_tr16(s + addr[b] + ks * 16 * RB);
      const v4i16 hi = lds_tr16(s + addr[b] + (ks * 16 + 4) * RB);
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = *(const float*)(s + addr[b] + (ks * 8 + e) * RB);
      return v;
    }
  }
};

// Over a whole workgroup, in a fixed order.
__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0;
  for (int i = 0; i < (int)blockDim.x / 64; ++i) s += lds[i];
  __syncthreads();
  return s;
}

// Sums of SUM_COLS columns, 16 threads each (ColumnSums).
constexpr int SUMS_LDS = 16 * (SUM_COLS + 1) * 4;
template <typename T> __device__ __forceinline__ float column_part(const T* p, long rows, int cols, int tr) {
  float s = 0.f;
#pragma unroll 8
  for (long r = tr; r < rows; r += 256 / SUM_COLS) s += elem_f(p[r * cols]);
  return s;
}
__device__ __forceinline__ void column_sums(const ColumnSums& a, int wg, char* smem) {
  float* const red = (float*)smem;
  const int tc = threadIdx.x % SUM_COLS, tr = threadIdx.x / SUM_COLS, col = wg * SUM_COLS + tc;
  float s = 0.f;
  if (col < a.cols)
    s = a.dt == BF16 ? column_part((const bf16_t*)a.src + col, a.rows, a.cols, tr)
                     : column_part((const float*)a.src + col, a.rows, a.cols, tr);
  red[tr * (SUM_COLS + 1) + tc] = s;
  __syncthreads();
  if (tr || col >= a.cols) return;
  s = 0.f;
#pragma unroll
  for (int r = 0; r < 256 / SUM_COLS; ++r) s += red[r * (SUM_COLS + 1) + tc];
  if (a.alpha) s *= a.alpha[0];
  a.out[col] = a.add ? a.out[col] + s : s;
}

// For up to FINISH_ROWS rows: the mean, and the bias gradient from the
// unrounded dlogits, FINISH_COLS columns per workgroup of 256 threads.  Each
// workgroup counts the rows for itself; the first one writes the mean.
constexpr int FINISH_LDS = 4 * 8 + 32 * (FINISH_COLS + 1) * 4;
__device__ __forceinline__ void loss_finish(const LossFinish& f, int wg, char* smem) {
  double* const lds = (double*)smem;
  float* const red = (float*)(smem + 4 * 8);
  const int t = threadIdx.x;
  double n = 0, s = 0;
  for (int r = t; r < f.rows; r += 256)
    if (label_ok(f.labels[r], f.classes)) {
      n += 1;
      if (wg == 0) s += f.loss[1 + r];
    }
  n = block_sum(n, lds);
  if (wg == 0) {
    s = block_sum(s, lds);
    if (t == 0) f.loss[0] = n > 0 ? (float)(s / n) : 0.f;
  }
  if (!f.db) return;
  const int tc = t % FINISH_COLS, tr = t / FINISH_COLS, col = wg * FINISH_COLS + tc;
  constexpr int LANES = 256 / FINISH_COLS;
  float c = 0.f;
  if (col < f.classes) {
#pragma unroll 4
    for (int r = tr; r < f.rows; r += LANES) c += label_ok(f.labels[r], f.classes) ? f.dz[(size_t)r * f.ld + col] : 0.f;
  }
  red[tr * (FINISH_COLS + 1) + tc] = c;
  __syncthreads();
  if (tr || col >= f.classes) return;
  c = 0.f;
#pragma unroll
  for (int r = 0; r < LANES; ++r) c += red[r * (FINISH_COLS + 1) + tc];
  c *= n > 0 ? (float)(f.scale / n) : 0.f;
  f.db[col] = f.add ? f.db[col] + c : c;
}

template <typename T, bool AKC, bool BKC, int WM, int WN, int FM, int FN> struct Shape {
  static constexpr int NW = WM * WN, BM = WM * FM * 32, BN = WN * FN * 32;
  typedef Tile<T, AKC, BM, NW> TA;
  typedef Tile<T, BKC, BN, NW> TB;
  static constexpr int STAGE = TA::BYTES + TB::BYTES;
  static constexpr int PIT = FN == 4 ? 152 : FN == 2 ? 88 : 56, HALF = FN * 16 + 16;  // floats per staged row; where its odd groups start
  static_assert(PIT % 16 == 8 && PIT >= HALF + FN * 16, "rows 4 apart lie half the banks apart");
  static constexpr int SMEM = 2 * STAGE > NW * 32 * PIT * 4 + BM * 12 ? 2 * STAGE : NW * 32 * PIT * 4 + BM * 12;
};

// A tile: WM x WN waves of (32 FM) x (32 FN).
//
// A K-tile is four steps of FM x FN matrix instructions (per 16 bytes of k).
// Between the instructions of a step the wave reads the fragments of the next
// one, so the matrix unit does not wait for LDS; the barrier of a K-tile comes
// before its last step, whose instructions cover the first reads of the next
// K-tile and the issue of the first loads of the one after that, into the stage
// that the barrier has freed; the other loads follow in the next step (64 KB in
// one step of 512 cycles were twice what the vector memory path takes: 870 ->
// 833 us at 8192^3).  A barrier waits for loads issued at least two steps ago.
//
// Bound by the matrix unit: 8192^3 bf16 1390 TFLOP/s (1.42 us a K-tile of 256 x
// 256, where 2.5 PFLOP/s would be 0.86), 4096^3 fp32 145 of a library product's
// 152; small products by the 10 .. 15 us that a tile's
// dispatch, first loads and epilogue take, and by rounds that do not fill.
//
// Workgroup `wg` of a product's tiles x splits.
template <typename T, bool AKC, bool BKC, int WM, int WN, int FM, int FN, int EPI>
__device__ __forceinline__ void product_tile(const GemmArgs& g, int wg, char* smem) {
  typedef Shape<T, AKC, BKC, WM, WN, FM, FN> S;
  typedef typename S::TA TA;
  typedef typename S::TB TB;
  constexpr int NW = S::NW, BM = S::BM, BN = S::BN, STAGE = S::STAGE, PIT = S::PIT, HALF = S::HALF;

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  // tiles in groups of 8 tile rows, column by column, dealt to the XCDs in
  // contiguous runs: neighbours share operand rows in one L2
  const int tiles = g.tiles_m * g.tiles_n;
  const int split = wg / tiles;
  int t = xcd_remap(wg - split * tiles, tiles);
  constexpr int GM = 8;
  const int group = t / (GM * g.tiles_n), first = group * GM, gm = min(GM, g.tiles_m - first);
  t -= group * GM * g.tiles_n;
  const int tm = first + t % gm, tn = t / gm;
  const int m0 = tm * BM, n0 = tn * BN;

  const int wm = wave / WN, wn = wave % WN;
  TA ta;
  TB tb;
  ta.init(wave, lane, g.lda, m0, g.M);
  tb.init(wave, lane, g.ldb, n0, g.N);
  Frags<T, AKC, BM, FM> fa;
  Frags<T, BKC, BN, FN> fb;
  fa.init(lane, wm * FM * 32);
  fb.init(lane, wn * FN * 32);

  f32x16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

  const int kt0 = split * g.kt_split, kt1 = min(g.kt_all, kt0 + g.kt_split);
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem);
  const uint32_t lds_a = lds0 + wave * TA::NI * 1024, lds_b = lds0 + TA::BYTES + wave * TB::NI * 1024;
  // Where the next K-tile to load starts in each operand, and the bytes from
  // there to the operand's end (a load past it reads zeros); advanced K-tile by
  // K-tile in scalar registers, in four parts that go between the matrix
  // instructions.  Past the last K-tile nothing is left: no traffic.
  const long step_a = AKC ? 128 : TA::BK * g.lda, step_b = BKC ? 128 : TB::BK * g.ldb;
  const char *pa, *pb;
  long left_a, left_b;
  int kt_next = kt0, kb_next = kt0;
  static_assert(TERMS == 3, "two places where B starts again");
  if (g.wrap && kb_next >= g.wrap) kb_next -= g.wrap;
  if (g.wrap && kb_next >= g.wrap) kb_next -= g.wrap;
  {
    const long at = (AKC ? (long)m0 * g.lda : (long)m0 * TA::ES) + kt0 * step_a;
    const long bt = (BKC ? (long)n0 * g.ldb : (long)n0 * TB::ES) + kb_next * step_b;
    pa = g.a + at;
    pb = g.b + bt;
    left_a = g.enda - at;
    left_b = g.endb - bt;
  }
  __amdgpu_buffer_rsrc_t ra, rb;
  auto clamp = [&](long left) {
    const int n = left > 0x7ffffff0L ? 0x7ffffff0 : (int)left;
    return (uint32_t)(kt_next < kt1 && left > 0 ? n : 0);
  };
  auto prepare = [&](int part) {
    if (part == 0) ra = make_rsrc(pa, clamp(left_a));
    if (part == 1) {
      pa += step_a;
      left_a -= step_a;
    }
    if (part == 2) rb = make_rsrc(pb, clamp(left_b));
    if (part == 3) {
      ++kb_next;
      const bool again = kb_next == g.wrap;
      const long d = again ? step_b - g.wrap * step_b : step_b;
      kb_next = again ? 0 : kb_next;
      pb += d;
      left_b -= d;
      ++kt_next;
    }
  };
  // before the last K-tile is loaded: it may hold less of K
  auto mask = [&](int kt) {
    if ((AKC || BKC) && kt == g.kt_all - 1) {
      ta.mask(wave, lane, g.kca - kt * 8);
      tb.mask(wave, lane, g.kcb - kt * 8);
    }
  };
  constexpr int NL = TA::NI + TB::NI;
  constexpr int NLA = NL / 2;  // loaded in a K-tile's last step; the others in the next one's first
  auto load = [&](int i, uint32_t stage) {
    if (i < TA::NI)
      ta.load(ra, lds_a + stage, i);
    else
      tb.load(rb, lds_b + stage, i - TA::NI);
  };
  typename Chunk<T>::type af[2][FM], bf[2][FN];
  // the matrix instructions of one step on fragments `cur`, with the reads of
  // step ks at s into the other set and, in between, what `with` says: 1: the
  // next loads are prepared; 2, 3: their first and second half
  auto step = [&](auto cur_, const char* s, auto ks_, auto with_, uint32_t stage) {
    constexpr int cur = decltype(cur_)::value, nxt = cur ^ 1, ks = decltype(ks_)::value, N = FM * FN;
    constexpr bool PREPARE = decltype(with_)::value == 1;
    constexpr int L0 = decltype(with_)::value == 2 ? 0 : decltype(with_)::value == 3 ? NLA : 0;
    constexpr int L1 = decltype(with_)::value == 2 ? NLA : decltype(with_)::value == 3 ? NL : 0;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      // fragments in the order in which the next step wants them
#pragma unroll
      for (int f = n * (FM + FN) / N; f < (n + 1) * (FM + FN) / N; ++f) {
        if (f < FN)
          bf[nxt][f] = fb.read(s + TA::BYTES, f, ks);
        else
          af[nxt][f - FN] = fa.read(s, f - FN, ks);
      }
      if constexpr (PREPARE) {
#pragma unroll
        for (int part = n * 4 / N; part < (n + 1) * 4 / N; ++part) prepare(part);
      }
#pragma unroll
      for (int l = L0 + n * (L1 - L0) / N; l < L0 + (n + 1) * (L1 - L0) / N; ++l) load(l, stage);
      mma32(af[cur][n / FN], bf[cur][n % FN], acc[n / FN][n % FN]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if (kt0 < kt1) {
    // the first K-tile, and of the second what a last step loads
    mask(kt0);
    for (int part = 0; part < 4; ++part) prepare(part);
#pragma unroll
    for (int i = 0; i < NL; ++i) load(i, 0);
    mask(kt0 + 1);
    for (int part = 0; part < 4; ++part) prepare(part);
#pragma unroll
    for (int i = 0; i < NLA; ++i) load(i, STAGE);
    wait_vmcnt<NLA>();  // the first K-tile has landed for this wave
    block_barrier();   // ... and for everyone
#pragma unroll
    for (int b = 0; b < FN; ++b) bf[0][b] = fb.read(smem + TA::BYTES, b, 0);
#pragma unroll
    for (int b = 0; b < FM; ++b) af[0][b] = fa.read(smem, b, 0);
    uint32_t stage = 0;
    for (int kt = kt0; kt < kt1; ++kt) {
      const char* s = smem + stage;
      step(Const<0>{}, s, Const<1>{}, Const<3>{}, stage ^ STAGE);
      step(Const<1>{}, s, Const<2>{}, Const<1>{}, 0);
      step(Const<0>{}, s, Const<3>{}, Const<0>{}, 0);
      mask(kt + 2);
      // vmcnt(0) lgkmcnt(0): the next K-tile has landed for this wave, and its
      // reads of this one are done; after the barrier so for everyone
      __builtin_amdgcn_s_waitcnt(0x0070);
      block_barrier();
      step(Const<1>{}, smem + (stage ^ STAGE), Const<0>{}, Const<2>{}, stage);
      stage ^= STAGE;
    }
  }
  wait_vmcnt<0>();  // what the last steps loaded (nothing is read, zeros are written)
  __syncthreads();  // everyone is done with the operand tiles

  // Each block of 32 rows goes through the wave's own LDS region, so that a
  // lane holds 8 consecutive columns of a row.  A staged row holds the even
  // groups of 4 columns, then the odd ones: a lane's two 16-byte reads, and the
  // rows' writes, meet every bank once.
  float* const q = (float*)(smem + wave * 32 * PIT * 4);
  constexpr int LPR = FN * 4;    // lanes per row
  constexpr int RPP = 64 / LPR;  // rows per pass
  constexpr int UN = 32 / RPP;   // passes of a block
  const int li = lane & 31, lh = lane >> 5;
  const int lr = lane % LPR, c8 = lr * 8, rr = lane / LPR;
  // A lane's columns: col .. col + 3 and colb .. colb + 3.  What is stored as
  // bf16 takes eight in a row; fp32 stores take four of each half of the wave's
  // columns, so that each instruction writes whole lines.
  const bool wide = EPI == EPI_OUT && (sizeof(T) == 4 || g.e.out_f32 || g.raw);
  const int col = n0 + wn * FN * 32 + (wide ? lr * 4 : c8), colb = wide ? col + FN * 16 : col + 4;
  const int qa = wide ? (lr >> 1) * 4 + (lr & 1 ? HALF : 0) : c8 / 2, qb = wide ? qa + FN * 8 : qa + HALF;
  const int wcol = (li & 3) + ((li >> 3) << 2) + (li & 4 ? HALF : 0);
  auto read = [&](int r, float (&v)[8]) {
    const float* s = q + r * PIT;
    const f32x4 a = *(const f32x4*)(s + qa), b = *(const f32x4*)(s + qb);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = a[j], v[4 + j] = b[j];
  };
  Columns cols{};
  float cs[8];
  if constexpr (EPI == EPI_OUT) {
    cols = columns_of(g.e, g.N, col, colb);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      cols.bias[j] = g.e.bias && col + j < g.N ? g.e.bias[col + j] : 0.f;
      cs[j] = 0.f;
    }
  }
  const bool edge = n0 + BN > g.N;  // columns past the end
  // Stores count as outstanding like loads, and a wait for a load waits for
  // every store before it: so what the rows take besides their sums is loaded
  // before the first store (the rows' labels and lse go through LDS), and what
  // is added to them a whole block ahead.
  struct RowInfo {
    int lab;
    float m, l2;  // row_lse's
  };
  static_assert(sizeof(RowInfo) == 12, "what SMEM counts");
  RowInfo* const info = (RowInfo*)(smem + NW * 32 * PIT * 4);
  const bool rows_have = EPI != EPI_OUT || g.e.labels;
  if (rows_have) {
    for (int r = threadIdx.x; r < BM; r += NW * 64) {
      const int row = m0 + r;
      RowInfo i{-1, 0.f, 0.f};
      if (row < g.M) {
        i.lab = g.e.labels[row];
        if constexpr (EPI == EPI_DLOGITS) {
          const float2 l = g.e.lse[row];
          i.m = l.x;
          i.l2 = l.y;
        }
      }
      info[r] = i;
    }
  }
  __syncthreads();
  __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0): the columns' values too
  auto stage_block = [&](auto bm_) {
    constexpr int bm = decltype(bm_)::value;
#pragma unroll
    for (int bn = 0; bn < FN; ++bn)
#pragma unroll
      for (int v = 0; v < 16; ++v) q[(8 * (v >> 2) + 4 * lh + (v & 3)) * PIT + bn * 16 + wcol] = acc[bm][bn][v];
  };
  Extra extra[UN];
  const bool adds = EPI == EPI_OUT && g.vec && !g.raw && (g.e.res || g.e.add);
  auto load_block = [&](int bm) {
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int row = m0 + (wm * FM + bm) * 32 + u * RPP + rr;
      extra[u] = load_extra<T>(g.e, g.M, g.N, row, col, colb);
    }
  };
  // Outputs from the tile's first row on, with 32-bit offsets: a lane's place in
  // the block's first row, computed once, and the rows' steps in scalar
  // registers.  Rows past the end lie past the buffer's, columns past it OOB.
  auto rows_from = [&](const void* p, long rows, uint32_t pitch) {
    const long left = (rows - m0) * pitch;
    return make_rsrc((const char*)p + (long)m0 * pitch, left > 0x7ffffff0L ? 0x7ffffff0u : left > 0 ? (uint32_t)left : 0u);
  };
  auto place = [&](int c, int cols, uint32_t pitch, int es) {
    return c < cols ? (uint32_t)(wm * FM * 32 + rr) * pitch + (uint32_t)(c * es) : OOB;
  };
  const int ys = g.e.out_f32 ? 4 : (int)sizeof(T);
  const uint32_t pitch_y = (uint32_t)g.e.ldy * ys, pitch_z = (uint32_t)g.N * (int)sizeof(T), pitch_p = (uint32_t)g.ldp * 4;
  const __amdgpu_buffer_rsrc_t yr = rows_from(g.e.y, EPI == EPI_DLOGITS ? g.e.rows_padded : g.M, pitch_y),
                               zr = rows_from(g.e.z, g.M, pitch_z),
                               pr = rows_from(g.partial + (size_t)split * g.M * g.ldp, g.M, pitch_p);
  const uint32_t at_y = place(col, EPI == EPI_DLOGITS ? (int)g.e.ldy : g.N, pitch_y, ys), at_yb = place(colb, g.N, pitch_y, ys),
                 at_z = place(col, g.N, pitch_z, (int)sizeof(T)), at_zb = place(colb, g.N, pitch_z, (int)sizeof(T)),
                 at_p = place(col, g.N, pitch_p, 4), at_pb = place(colb, g.N, pitch_p, 4);
  __amdgpu_buffer_rsrc_t mr0 = yr, mr1 = yr;  // the further terms
  if (EPI == EPI_DLOGITS && g.e.more) {
    static_assert(TERMS == 3, "two further terms");
    mr0 = rows_from(g.e.more, g.e.rows_padded, pitch_y);
    mr1 = rows_from(g.e.more + (size_t)g.e.rows_padded * g.e.ldy, g.e.rows_padded, pitch_y);
  }
  if (adds) load_block(0);
  // The accumulators' registers need constant indexes, the rest does not: one
  // copy of it, which stays in the instruction cache.
#pragma unroll 1
  for (int bm = 0; bm < FM; ++bm) {
    const int row0 = m0 + (wm * FM + bm) * 32;
    if (bm == 0) stage_block(Const<0>{});
    if constexpr (FM >= 2) {
      if (bm == 1) stage_block(Const<1>{});
    }
    if constexpr (FM == 4) {
      if (bm == 2) stage_block(Const<2>{});
      if (bm == 3) stage_block(Const<3>{});
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): this wave's LDS writes are done
    __builtin_amdgcn_wave_barrier();
    if constexpr (EPI == EPI_OUT) {
      if (g.raw) {
        float v[UN][8];
#pragma unroll
        for (int u = 0; u < UN; ++u) read(u * RPP + rr, v[u]);
#pragma unroll
        for (int u = 0; u < UN; ++u) {
          const uint32_t step = (uint32_t)(bm * 32 + u * RPP) * pitch_p;
          buf_store4<false>(pr, at_p + step, v[u]);
          buf_store4<false>(pr, at_pb + step, v[u] + 4);
        }
      } else if (g.vec) {
        float v[UN][8];
        bool live[UN];
#pragma unroll
        for (int u = 0; u < UN; ++u) {
          const int r = u * RPP + rr;
          read(r, v[u]);
          live[u] = !rows_have || label_ok(info[row0 + r - m0].lab, g.e.classes);
        }
        auto put = [&](__amdgpu_buffer_rsrc_t b, uint32_t o, uint32_t ob, uint32_t pitch, int u, const float(&w)[8]) {
          const uint32_t step = (uint32_t)(bm * 32 + u * RPP) * pitch;
          if (wide) {
            buf_store4<true>(b, o + step, w);
            buf_store4<true>(b, ob + step, w + 4);
          } else {
            buf_store8h<true>(b, o + step, w);
          }
        };
        epi_out<T, UN>(
            g.e, v, cols, extra, live, [&](int u, const float(&w)[8]) { put(zr, at_z, at_zb, pitch_z, u, w); },
            [&](int u, const float(&w)[8]) { put(yr, at_y, at_yb, pitch_y, u, w); },
            // the next block's before this one's stores, which its wait then leaves alone
            [&] {
              if (adds && bm + 1 < FM) load_block(bm + 1);
            });
      } else {
#pragma unroll 1
        for (int u = 0; u < UN; ++u) {
          const int r = u * RPP + rr, row = row0 + r;
          const bool live = !rows_have || label_ok(info[row - m0].lab, g.e.classes);
          float v[8];
          read(r, v);
          if (row < g.M) epi_out_any<T>(g.e, g.N, row, col, colb, v, cols, live);
        }
      }
    } else {
      float vs[UN][8];
      RowInfo ris[UN];
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        read(u * RPP + rr, vs[u]);
        ris[u] = info[row0 + u * RPP + rr - m0];
      }
      // Each step for all rows before the next: their chains of dependent
      // instructions overlap, and what few rows need is one branch for all.
      bool hit = false, dead = false;
      uint32_t at[UN];
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        at[u] = (uint32_t)ris[u].lab - (uint32_t)(g.e.col0 + col);
        if (!label_ok(ris[u].lab, g.e.classes)) {
          dead = true;
          at[u] = 8u;
        }
        hit |= at[u] < 8u;
#pragma unroll
        for (int j = 0; j < 8; ++j) vs[u][j] += cols.bias[j];
      }
      hit = __any(hit);
      dead = __any(dead);
      if constexpr (EPI == EPI_LSE) {
        static_assert(EPI != EPI_LSE || FN * 32 % STAT_COLS == 0, "whole groups of columns");
        constexpr int LPG = STAT_COLS / 8;  // lanes per group
        if (edge) {
#pragma unroll
          for (int u = 0; u < UN; ++u)
#pragma unroll
            for (int j = 0; j < 8; ++j) vs[u][j] = col + j < g.N ? vs[u][j] : -INFINITY;
        }
        float m[UN], s[UN];
#pragma unroll
        for (int u = 0; u < UN; ++u) {
          const float(&v)[8] = vs[u];
          m[u] = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
        }
#pragma unroll
        for (int d = 1; d < LPG; d <<= 1)
#pragma unroll
          for (int u = 0; u < UN; ++u) m[u] = fmaxf(m[u], lane_xor(m[u], d));
#pragma unroll
        for (int u = 0; u < UN; ++u) {
          const float ms = m[u] == -INFINITY ? 0.f : m[u];
          float x[8];  // their sum is NaN where a value is (fmaxf passed over it)
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] = exp_fast(vs[u][j] - ms);
          s[u] = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
        }
#pragma unroll
        for (int d = 1; d < LPG; d <<= 1)
#pragma unroll
          for (int u = 0; u < UN; ++u) s[u] += lane_xor(s[u], d);
        if (c8 % STAT_COLS == 0 && col < g.N) {
#pragma unroll
          for (int u = 0; u < UN; ++u) {
            const int row = row0 + u * RPP + rr;
            if (row < g.M) g.e.stats[(size_t)row * g.e.nstat + g.e.stat0 + col / STAT_COLS] = make_float2(m[u], s[u]);
          }
        }
        if (hit) {
#pragma unroll
          for (int u = 0; u < UN; ++u) {
            if (at[u] < 8u) {
              float z = vs[u][0];
#pragma unroll
              for (int j = 1; j < 8; ++j) z = at[u] == (uint32_t)j ? vs[u][j] : z;
              g.e.zlab[row0 + u * RPP + rr] = z;
            }
          }
        }
      } else {
#pragma unroll
        for (int u = 0; u < UN; ++u)
#pragma unroll
          for (int j = 0; j < 8; ++j) vs[u][j] = row_prob(vs[u][j], make_float2(ris[u].m, ris[u].l2));
        if (hit) {
#pragma unroll
          for (int u = 0; u < UN; ++u)
#pragma unroll
            for (int j = 0; j < 8; ++j) vs[u][j] -= at[u] == (uint32_t)j ? 1.f : 0.f;
        }
        if (edge || dead) {
#pragma unroll
          for (int u = 0; u < UN; ++u)
#pragma unroll
            for (int j = 0; j < 8; ++j)
              vs[u][j] = label_ok(ris[u].lab, g.e.classes) && col + j < g.N ? vs[u][j] : 0.f;
        }
        if (g.e.colsum) {
#pragma unroll
          for (int u = 0; u < UN; ++u)
#pragma unroll
            for (int j = 0; j < 8; ++j) cs[j] += vs[u][j];
        }
#pragma unroll
        for (int u = 0; u < UN; ++u) {
          const uint32_t o = at_y + (uint32_t)(bm * 32 + u * RPP) * pitch_y;
          if constexpr (sizeof(T) == 4) {
            buf_store4<false>(yr, o, vs[u]);
            buf_store4<false>(yr, o + 16, vs[u] + 4);
          } else {
            buf_store8h<false>(yr, o, vs[u]);
          }
        }
        if constexpr (sizeof(T) == 2) {
          if (g.e.more) {
#pragma unroll
            for (int t = 0; t < TERMS - 1; ++t)
#pragma unroll
              for (int u = 0; u < UN; ++u) {
#pragma unroll
                for (int j = 0; j < 8; ++j) vs[u][j] -= bf16_to_f32(f32_to_bf16(vs[u][j]));
                buf_store8h<false>(t ? mr1 : mr0, at_y + (uint32_t)(bm * 32 + u * RPP) * pitch_y, vs[u]);
              }
          }
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
    if constexpr (EPI == EPI_DLOGITS) {
      static_assert(FM * 32 % COLSUM_ROWS == 0 || EPI != EPI_DLOGITS, "whole groups of rows");
      if (((bm + 1) * 32) % COLSUM_ROWS == 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
#pragma unroll
          for (int d = LPR; d < 64; d <<= 1) cs[j] += __shfl_xor(cs[j], d);
        }
        const int row = row0 + 32 - COLSUM_ROWS;
        if (g.e.colsum && rr == 0 && row < g.M) {
          float* out = g.e.colsum + (size_t)(row / COLSUM_ROWS) * g.N + col;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (col + j < g.N) out[j] = cs[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) cs[j] = 0.f;
      }
    }
  }
}

template <typename T, bool AKC, bool BKC, int WM, int WN, int FM, int FN, int EPI>
__global__ __launch_bounds__(WM* WN * 64, FM == 4 ? 1 : FM == 2 ? 2 : 4) void product_kernel(GemmArgs g) {
  __shared__ __align__(1024) char smem[Shape<T, AKC, BKC, WM, WN, FM, FN>::SMEM];
  product_tile<T, AKC, BKC, WM, WN, FM, FN, EPI>(g, blockIdx.x, smem);
}

// The two products of a layer's gradients in one launch, source gradient
// first: neither leaves the chip half empty while the other waits.
// What is left of the bias gradient (ColumnSums: 5 us by itself) or of a loss
// (LossFinish) rides along in further workgroups.
struct PairArgs {
  GemmArgs dx, dw;
  int wgs_dx, wgs, wgs_sums;  // workgroups: of dx, of both products, and with the sums'
  ColumnSums sums;
  LossFinish finish;
};
template <typename T, int FM, int FN>
__global__ __launch_bounds__(256, FM == 4 ? 1 : FM == 2 ? 2 : 4) void product_pair_kernel(PairArgs p) {
  constexpr int S1 = Shape<T, true, false, 2, 2, FM, FN>::SMEM, S2 = Shape<T, false, false, 2, 2, FM, FN>::SMEM;
  __shared__ __align__(1024) char smem[S1 > S2 ? S1 : S2];
  if ((int)blockIdx.x < p.wgs_dx)
    product_tile<T, true, false, 2, 2, FM, FN, EPI_OUT>(p.dx, blockIdx.x, smem);
  else if ((int)blockIdx.x < p.wgs)
    product_tile<T, false, false, 2, 2, FM, FN, EPI_OUT>(p.dw, (int)blockIdx.x - p.wgs_dx, smem);
  else if ((int)blockIdx.x < p.wgs_sums)
    column_sums(p.sums, (int)blockIdx.x - p.wgs, smem);
  else
    loss_finish(p.finish, (int)blockIdx.x - p.wgs_sums, smem);
}

// Adds the partial sums of a split product in order and finishes them.
template <typename T> __global__ __launch_bounds__(256) void product_reduce_kernel(GemmArgs g) {
  const int n8 = (int)(g.ldp / 8);
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  if (i >= (long)g.M * n8) return;
  const int row = (int)(i / n8), col = (int)(i - (long)row * n8) * 8;
  float v[8];
  const float* p = g.partial + (size_t)row * g.ldp + col;
  const size_t step = (size_t)g.M * g.ldp;
  load8<float>(p, v);
  for (int s = 1; s < g.splits; s += 4) {  // four loads under way, added in order
    float u[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) load8<float>(p + min(s + i, g.splits - 1) * step, u[i]);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += s + i < g.splits ? u[i][j] : 0.f;
  }
  const bool live = !g.e.labels || label_ok(g.e.labels[row], g.e.classes);
  const Columns c = columns_of(g.e, g.N, col, col + 4);
  if (!g.vec) return epi_out_any<T>(g.e, g.N, row, col, col + 4, v, c, live);
  Extra x[1];
  float v1[1][8];
  if (g.e.res || g.e.add) x[0] = load_extra<T>(g.e, g.M, g.N, row, col, col + 4);
#pragma unroll
  for (int j = 0; j < 8; ++j) v1[0][j] = v[j];
  const size_t o = (size_t)row * g.N + col, oy = (size_t)row * g.e.ldy + col;
  epi_out<T, 1>(
      g.e, v1, c, x, {live}, [&](int, const float(&w)[8]) { store8<T>((T*)g.e.z + o, w); },
      [&](int, const float(&w)[8]) {
        if (g.e.out_f32)
          store8<float>((float*)g.e.y + oy, w);
        else
          store8<T>((T*)g.e.y + oy, w);
      },
      [] {});
}

// ------------------------------------------------------------------ plans
//
// Tiles of 256 x 256 (bf16), 128 x 128, or 64 x 64 (fp32, whose matrix
// instructions are slow enough for the smaller tile's loads), and the cut of
// the K range, from a model of the time in us that follows what was measured
// (MI355X, 24 products of 128 .. 4096 rows, 256 .. 32768 of k).  A K-tile takes
//   256: 1.42, and 10 per tile; one workgroup per CU
//   128: bf16 0.44 while there is one workgroup per CU and 1.0 at two, fp32
//        1.95 times the workgroups per CU; 5 per tile
//   64:  0.55 times the workgroups per CU; 4 per tile
// and a cut costs the second launch, 4, and its partial sums' bytes at 6 TB/s
// (also where the sums are left raw and their reader adds them up: product_splits
// takes the same plan).
enum { TILE_128 = 0, TILE_256 = 1, TILE_64 = 2 };
struct Plan {
  int tile, splits, kt_split;
  double t;
};
inline long div_up(long a, long b) { return (a + b - 1) / b; }
inline int tile_rows(int tile) { return tile == TILE_256 ? 256 : tile == TILE_64 ? 64 : 128; }
inline long tiles_of(int tile, int M, int N) { return div_up(M, tile_rows(tile)) * div_up(N, tile_rows(tile)); }
inline bool tile_ok(int tile, int dt, int epi) { return tile == TILE_128 || (tile == TILE_256 ? dt == BF16 : dt == F32 && epi == EPI_OUT); }
inline int ktiles(int dt, int K) { return (int)div_up(K, dt == BF16 ? 64 : 32); }

// Workgroups that run at once, and the time of one of `per` K-tiles while `n`
// are there.
inline int slots_of(int tile, int dt) { return tile == TILE_128 && dt == BF16 ? 512 : 256; }
inline double wg_time(int tile, int dt, long per, long n) {
  if (tile == TILE_256) return per * 1.42 + 10;
  if (tile == TILE_64) return per * 0.55 + 4;
  if (dt == F32) return per * 1.95 + 5;
  return per * (n <= 256 ? 0.44 : n >= 512 ? 1.0 : 0.44 + (n - 256) / 256.0 * 0.56) + 5;
}
inline double cut_time(int s, int M, int N) { return s > 1 ? 4 + s * (double)M * N * 8 / 6e6 : 0; }

inline Plan plan_product(int dt, int M, int N, int K, int epi) {
  const int kt = ktiles(dt, K);
  Plan best{TILE_128, 1, kt, 1e30};
  for (int tile = 0; tile < 3; ++tile) {
    if (!tile_ok(tile, dt, epi)) continue;
    const long tiles = tiles_of(tile, M, N);
    for (int s = 1; s <= 32 && s <= kt && (s == 1 || epi == EPI_OUT); ++s) {
      const long n = tiles * s, per = div_up(kt, s);
      if (s > 1 && n > 1024) break;
      const double t = div_up(n, slots_of(tile, dt)) * wg_time(tile, dt, per, n) + cut_time(s, M, N);
      if (t < best.t) best = Plan{tile, (int)div_up(kt, per), (int)per, t};
    }
  }
  return best;
}

// The same for two products in one launch (of one tile): as long as the longer
// workgroup, or as all of them over the slots and half of a shorter one at the
// end (250 + 256 tiles of 256 x 256: 251 us, one after the other 228).
struct PairPlan {
  Plan a, b;
  double t;
};
inline PairPlan plan_pair(int dt, int Ma, int Na, int Ka, int Mb, int Nb, int Kb) {
  static const int cuts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
  const int ka = ktiles(dt, Ka), kb = ktiles(dt, Kb);
  PairPlan best{{}, {}, 1e30};
  for (int tile = 0; tile < 3; ++tile) {
    if (!tile_ok(tile, dt, EPI_OUT)) continue;
    const long ta = tiles_of(tile, Ma, Na), tb = tiles_of(tile, Mb, Nb);
    const int slots = slots_of(tile, dt);
    for (int sa : cuts)
      for (int sb : cuts) {
        if (sa > ka || sb > kb) continue;
        const long na = ta * sa, nb = tb * sb, pa = div_up(ka, sa), pb = div_up(kb, sb);
        if ((sa > 1 && na > 1024) || (sb > 1 && nb > 1024)) continue;
        const double da = wg_time(tile, dt, pa, na + nb), db = wg_time(tile, dt, pb, na + nb);
        double t = da > db ? da : db;
        const double lo = da < db ? da : db;
        const double all = (na * da + nb * db) / slots + (na + nb > slots ? 0.5 * lo : 0);
        if (all > t) t = all;
        t += cut_time(sa, Ma, Na) + cut_time(sb, Mb, Nb);
        if (t < best.t) best = PairPlan{{tile, (int)div_up(ka, pa), (int)pa, t}, {tile, (int)div_up(kb, pb), (int)pb, t}, t};
      }
  }
  return best;
}
// One launch, unless the two products by themselves are faster (a launch: 3).
inline bool pair_pays(int dt, const PairPlan& p, int Ma, int Na, int Ka, int Mb, int Nb, int Kb) {
  return p.t < plan_product(dt, Ma, Na, Ka, EPI_OUT).t + plan_product(dt, Mb, Nb, Kb, EPI_OUT).t + 3;
}
// Up to SKINNY_ROWS rows: the kernel without LDS (skinny_kernel), in blocks of
// 16 mt rows, against tiles (and, for odd row lengths, the copies that those
// need).  Measured, in us, at 16 / 64 / 128 / 256 rows: bf16 1000 x 776 (K x N)
// 6 / 6 / 5 / 6 against 11; 1001 x 777 6 / 6 / 8 / 13 against 16 .. 17; 4096 x
// 1000 9 / 9 / 13 / 21 against 13 .. 16; 4096 x 4096 9 / 20 / 38 / 73 against
// 14 / 15 / 18 / 23; fp32 1001 x 777 5 / 6 / 7 / 10 against 16 .. 20, 4096 x
// 4096 16 / 39 / 75 / 145 against 26 / 28 / 48 / 83.  A workgroup reads 16 rows
// of B and its rows of A, 16 bytes of 16 rows per instruction, and both pass
// through the caches: the time goes with the bytes of a row, and with the
// workgroups per CU (which do not overlap much where rows are long, hence half
// of the rounded number).  bf16 rows that start inside a 4-byte word take 2.5 to
// 3.5 times as long.
struct SkinnyPlan {
  int mt;  // blocks of 16 rows per workgroup
  double t;
};
inline SkinnyPlan plan_skinny(int dt, int M, int N, int K) {
  const double kb = (dt == BF16 ? 2.0 : 4.0) * K / 2048;
  SkinnyPlan best{1, 1e30};
  for (int mt = 1; mt <= 4; mt *= 2) {
    const int r = M < 16 * mt ? M : 16 * mt;
    const double wgs = (double)(div_up(N, 16) * div_up(M, 16 * mt)) / 256;
    const double rounds = wgs <= 1 ? 1 : 0.5 * (wgs + (double)(long)(wgs + 0.999));
    const double odd = dt == BF16 && K % 2 ? 2.4 + 0.07 * (r < 16 ? r : 16) : 1;
    const double per = odd * kb * (r <= 16 ? 1.37 + 0.03 * r : 1.1 + 0.054 * r), least = 0.25 + 0.15 * mt;
    const double t = 1.5 + rounds * (per > least ? per : least);
    if (t < best.t) best = SkinnyPlan{mt, t < 5 ? 5 : t};
    if (M <= 16 * mt) break;
  }
  return best;
}
// copied: the tiles' operands are needed for other products as well.
inline bool skinny_pays(int dt, int M, int N, int K, bool copied) {
  if (M > SKINNY_ROWS) return false;
  const double es = dt == BF16 ? 2 : 4, bytes = es * N * K;
  double tiles = plan_product(dt, M, N, K, EPI_OUT).t;
  if (tiles < 5 + bytes / 5.3e6) tiles = 5 + bytes / 5.3e6;
  if (!copied && K % (dt == BF16 ? 8 : 4)) tiles += 4 + 2 * es * ((double)M + N) * K / 5e6;
  return plan_skinny(dt, M, N, K).t < tiles;
}

inline size_t partial_bytes_of(const Plan& p, int M, int N) {
  return p.splits > 1 ? (size_t)p.splits * M * (((size_t)N + 7) / 8 * 8) * 4 : 0;
}

// --------------------------------------------------------------- launches
template <typename T> GemmArgs args_of(const Product& p, const Plan& pl, float* partial) {
  constexpr int ES = (int)sizeof(T), VEC = TypeInfo<T>::VEC;
  const int bm = tile_rows(pl.tile);
  GemmArgs g{};
  const long kb = p.kb ? p.kb : p.K;
  g.a = (const char*)p.a.p;
  g.b = (const char*)p.b.p;
  g.lda = p.a.ld * ES;
  g.ldb = p.b.ld * ES;
  g.enda = (p.a.kc ? (long)p.M : (long)p.K) * g.lda;
  g.endb = (p.b.kc ? (long)p.N : kb) * g.ldb;
  g.M = p.M;
  g.N = p.N;
  g.kca = g.kcb = (p.K + VEC - 1) / VEC;
  g.kt_all = ktiles(p.dt, p.K);
  g.kt_split = pl.kt_split;
  g.splits = pl.splits;
  g.wrap = p.wrap / TypeInfo<T>::BK;
  g.tiles_m = (p.M + bm - 1) / bm;
  g.tiles_n = (p.N + bm - 1) / bm;
  g.partial = partial;
  g.ldp = ((long)p.N + 7) / 8 * 8;
  g.raw = p.raw || g.splits > 1;
  g.vec = p.N % 8 == 0;
  g.e = p.e;
  if (!g.e.ldy) g.e.ldy = p.N;
  return g;
}

template <typename T> hipError_t launch_reduce(const Product& p, const GemmArgs& g, hipStream_t st) {
  if (g.splits == 1 || p.raw) return hipSuccess;
  TraceScope ts("product_reduce_kernel", st, 4.0 * (g.splits + 1) * p.M * p.N, WORK_BYTE);
  hipLaunchKernelGGL(product_reduce_kernel<T>, dim3((unsigned)(((long)p.M * (g.ldp / 8) + 255) / 256)), dim3(256), 0, st, g);
  return hipGetLastError();
}

inline long wgs_of(const GemmArgs& g) { return (long)g.tiles_m * g.tiles_n * g.splits; }

template <typename T, bool AKC, bool BKC, int EPI> hipError_t launch_tiles(const Product& p, const GemmArgs& g, int tile, hipStream_t st) {
  const dim3 grid((unsigned)wgs_of(g));
  TraceScope ts(p.name, st, p.flops, WORK_FLOP);
  constexpr bool F = sizeof(T) == 4;
  if (!F && tile == TILE_256)
    hipLaunchKernelGGL((product_kernel<T, AKC, BKC, 2, 2, F ? 2 : 4, F ? 2 : 4, EPI>), grid, dim3(256), 0, st, g);
  else if (F && EPI == EPI_OUT && tile == TILE_64)
    hipLaunchKernelGGL((product_kernel<T, AKC, BKC, 2, 2, F && EPI == EPI_OUT ? 1 : 2, F && EPI == EPI_OUT ? 1 : 2, EPI>), grid,
                       dim3(256), 0, st, g);
  else
    hipLaunchKernelGGL((product_kernel<T, AKC, BKC, 2, 2, 2, 2, EPI>), grid, dim3(256), 0, st, g);
  return hipGetLastError();
}

template <typename T> hipError_t launch_product_t(const Product& p, float* partial, hipStream_t st) {
  const Plan pl = plan_product(p.dt, p.M, p.N, p.K, p.epi);
  const GemmArgs g = args_of<T>(p, pl, partial);
  hipError_t e = hipErrorNotSupported;
  if (p.epi == EPI_OUT) {
    if (p.a.kc && p.b.kc) e = launch_tiles<T, true, true, EPI_OUT>(p, g, pl.tile, st);
    if (p.a.kc && !p.b.kc) e = launch_tiles<T, true, false, EPI_OUT>(p, g, pl.tile, st);
    if (!p.a.kc && !p.b.kc) e = launch_tiles<T, false, false, EPI_OUT>(p, g, pl.tile, st);
  } else if (p.a.kc && p.b.kc) {
    e = p.epi == EPI_LSE ? launch_tiles<T, true, true, EPI_LSE>(p, g, pl.tile, st)
                         : launch_tiles<T, true, true, EPI_DLOGITS>(p, g, pl.tile, st);
  }
  return e == hipSuccess ? launch_reduce<T>(p, g, st) : e;
}

template <typename T>
hipError_t launch_pair_t(const Product& dx, const Product& dw, const ColumnSums* sums, const LossFinish* finish,
                         float* partial, hipStream_t st) {
  const PairPlan pl = plan_pair(dx.dt, dx.M, dx.N, dx.K, dw.M, dw.N, dw.K);
  if (!pair_pays(dx.dt, pl, dx.M, dx.N, dx.K, dw.M, dw.N, dw.K)) {
    hipError_t e = sums ? launch_column_sums(*sums, st) : hipSuccess;
    if (e == hipSuccess && finish) e = launch_loss_finish(*finish, st);
    if (e == hipSuccess) e = launch_product_t<T>(dx, partial, st);
    return e == hipSuccess ? launch_product_t<T>(dw, partial, st) : e;
  }
  PairArgs a{};
  a.dx = args_of<T>(dx, pl.a, partial);
  a.dw = args_of<T>(dw, pl.b, partial + partial_bytes_of(pl.a, dx.M, dx.N) / 4);
  a.wgs_dx = (int)wgs_of(a.dx);
  a.wgs = (int)(wgs_of(a.dx) + wgs_of(a.dw));
  a.wgs_sums = a.wgs + (sums ? (int)sums_wgs(*sums) : 0);
  if (sums) a.sums = *sums;
  if (finish) a.finish = *finish;
  const dim3 grid((unsigned)a.wgs_sums + (finish ? finish_wgs(*finish) : 0u));
  {
    TraceScope ts("product_pair_kernel", st, dx.flops + dw.flops, WORK_FLOP);
    constexpr bool F = sizeof(T) == 4;
    if (!F && pl.a.tile == TILE_256)
      hipLaunchKernelGGL((product_pair_kernel<T, F ? 2 : 4, F ? 2 : 4>), grid, dim3(256), 0, st, a);
    else if (F && pl.a.tile == TILE_64)
      hipLaunchKernelGGL((product_pair_kernel<T, F ? 1 : 2, F ? 1 : 2>), grid, dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL((product_pair_kernel<T, 2, 2>), grid, dim3(256), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const hipError_t e = launch_reduce<T>(dx, a.dx, st);
  return e == hipSuccess ? launch_reduce<T>(dw, a.dw, st) : e;
}

}  // namespace

}  // namespace singa
