// dense_aux.hip -- the dense product of few rows, and the kernels around the
// products: operands laid out for the tiles, the gradient through an
// activation, column sums, and the rows of a softmax cross-entropy.
#include "dense_gemm.h"

namespace singa {

namespace {

// ------------------------------------------------- product of few rows
//
// A workgroup takes 16 rows of B (the weights) and up to 16 MT rows of A,
// straight into registers: v_mfma_f32_16x16x32_bf16 (or four v_mfma_f32_16x16x4_f32) takes
// 16 bytes of a row from each lane, 64 consecutive bytes of a row per step, so
// neither operand needs LDS and any row start will do (ALIGNED: the rows start
// at 16-byte boundaries; otherwise the same loads without that promise, and the
// end of a row element by element).  The waves share the K range and add their
// sums through LDS.  Bound by the bytes of B where A is one block of rows (4096
// x 32000 bf16, one row: 6.3 TB/s), else by what the caches deliver; U steps (U
// x 64 bytes of 16 rows) are in flight per wave.
typedef float f32x4v __attribute__((ext_vector_type(4)));

__device__ __forceinline__ void mma16(const bf16x8& a, const bf16x8& b, f32x4v& c) {
  c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ void mma16(const f32x4& a, const f32x4& b, f32x4v& c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
}

// 16 bytes of a row from element k, all of them within it
template <typename T, bool ALIGNED> __device__ __forceinline__ typename Chunk<T>::type row_chunk(const T* row, int k) {
  typename Chunk<T>::type c;
  if constexpr (ALIGNED)
    c = *(const typename Chunk<T>::type*)(row + k);
  else
    __builtin_memcpy(&c, row + k, 16);
  return c;
}
// the same near the row's end: elements from K on are zero
template <typename T, bool ALIGNED> __device__ __forceinline__ typename Chunk<T>::type row_end(const T* row, int k, int K) {
  constexpr int VEC = TypeInfo<T>::VEC;
  if (k + VEC <= K) return row_chunk<T, ALIGNED>(row, k);
  union { typename Chunk<T>::type c; T e[VEC]; } u;
#pragma unroll
  for (int j = 0; j < VEC; ++j) u.e[j] = k + j < K ? row[k + j] : zero_elem<T>();
  return u.c;
}

// Eight waves share the K range: of 4 / 8 / 16 they took, for one row, bf16
// 4096 x 4096 7.4 / 6.9 / 7.1 us, 32000 x 4096 44.4 / 41.9 / 42.5, and fp32
// 50000 x 2048 76.8 / 69 / 67.6.
constexpr int SKINNY_WAVES = 8;

template <typename T, bool ALIGNED, int MT, int EPI>
__global__ __launch_bounds__(SKINNY_WAVES * 64) void skinny_kernel(const T* __restrict__ x, const T* __restrict__ w, int M,
                                                                   int N, int K, Epilogue e) {
  constexpr int VEC = TypeInfo<T>::VEC, U = MT <= 2 ? 8 : 4, STEP = 4 * VEC;
  __shared__ float red[SKINNY_WAVES][MT * 16][16];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, li = lane & 15, kq = lane >> 4;
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * MT * 16;
  // rows past the end read the last one; their results are not used
  const T* wr = w + (size_t)min(n0 + li, N - 1) * K;
  const T* xr[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) xr[m] = x + (size_t)min(m0 + m * 16 + li, M - 1) * K;
  f32x4v acc[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) acc[m] = f32x4v{0.f, 0.f, 0.f, 0.f};
  typedef typename Chunk<T>::type C;
  const int full = K / (STEP * U);  // runs of U whole steps
  // Rows a multiple of 16 KB apart start in the same memory channels: with the
  // chip full of workgroups, each starts at another run (one row, fp32 4096 x
  // 4096 17.4 -> 11.2 us, bf16 4096 x 8192 18.5 -> 12.8; at other pitches that
  // cost up to a quarter, 32000 x 4096 bf16 42 -> 52).
  const int rot = (size_t)K * sizeof(T) % 16384 == 0 && N >= 4096 ? (int)(blockIdx.x % (unsigned)full) : 0;
  for (int it = wave; it < full; it += SKINNY_WAVES) {
    const int run = it + rot < full ? it + rot : it + rot - full;
    const int k = run * STEP * U + kq * VEC;
    C wc[U], xc[MT][U];
#pragma unroll
    for (int u = 0; u < U; ++u) wc[u] = row_chunk<T, ALIGNED>(wr, k + u * STEP);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int u = 0; u < U; ++u) xc[m][u] = row_chunk<T, ALIGNED>(xr[m], k + u * STEP);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int m = 0; m < MT; ++m) mma16(wc[u], xc[m][u], acc[m]);
  }
  // the remaining steps one by one; a lane past the end adds zeros
  for (int k0 = full * STEP * U + wave * STEP; k0 < K; k0 += SKINNY_WAVES * STEP) {
    const int k = k0 + kq * VEC;
    C wc{}, xc[MT]{};
    if (k < K) {
      wc = row_end<T, ALIGNED>(wr, k, K);
#pragma unroll
      for (int m = 0; m < MT; ++m) xc[m] = row_end<T, ALIGNED>(xr[m], k, K);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) mma16(wc, xc[m], acc[m]);
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) *(f32x4v*)&red[wave][m * 16 + li][kq * 4] = acc[m];
  __syncthreads();
  for (int idx = threadIdx.x; idx < MT * 256; idx += SKINNY_WAVES * 64) {
    const int row = m0 + (idx >> 4), c = idx & 15, col = n0 + c;
    float v = 0.f;
#pragma unroll
    for (int s = 0; s < SKINNY_WAVES; ++s) v += red[s][idx >> 4][c];
    const bool in = row < M && col < N;
    if (e.bias && in) v += e.bias[col];
    if constexpr (EPI == EPI_OUT) {
      if (!in) continue;
      const size_t o = (size_t)row * N + col;
      if (e.z) store_out<T>((T*)e.z + o, v);
      if (e.act) v = act_f<T>(v, e.act);
      if (e.res) v += elem_f(((const T*)e.res)[o]);
      if (e.out_f32)
        ((float*)e.y)[(size_t)row * e.ldy + col] = v;
      else
        store_out<T>((T*)e.y + (size_t)row * e.ldy + col, v);
    } else {
      const float z = v;
      v = in ? v : -INFINITY;
      float m = v;
#pragma unroll
      for (int d = 1; d < 16; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
      float s = exp_fast(v - (m == -INFINITY ? 0.f : m));
#pragma unroll
      for (int d = 1; d < 16; d <<= 1) s += __shfl_xor(s, d);
      if (row < M) {
        if (c == 0) e.stats[(size_t)row * e.nstat + e.stat0 + blockIdx.x] = make_float2(m, s);
        if (in && e.labels[row] == e.col0 + col) e.zlab[row] = z;
      }
    }
  }
}

template <typename T, bool ALIGNED, int EPI> hipError_t skinny_rows(const Product& p, hipStream_t st) {
  const int mt = plan_skinny(p.dt, p.M, p.N, p.K).mt;
  const dim3 grid((unsigned)((p.N + 15) / 16), (unsigned)((p.M + 16 * mt - 1) / (16 * mt))), block(SKINNY_WAVES * 64);
  const T *x = (const T*)p.a.p, *w = (const T*)p.b.p;
  Epilogue e = p.e;
  if (!e.ldy) e.ldy = p.N;
  TraceScope ts(p.name, st, p.flops, WORK_FLOP);
  switch (mt) {
    case 1: hipLaunchKernelGGL((skinny_kernel<T, ALIGNED, 1, EPI>), grid, block, 0, st, x, w, p.M, p.N, p.K, e); break;
    case 2: hipLaunchKernelGGL((skinny_kernel<T, ALIGNED, 2, EPI>), grid, block, 0, st, x, w, p.M, p.N, p.K, e); break;
    default: hipLaunchKernelGGL((skinny_kernel<T, ALIGNED, 4, EPI>), grid, block, 0, st, x, w, p.M, p.N, p.K, e); break;
  }
  return hipGetLastError();
}

template <typename T> hipError_t skinny_t(const Product& p, hipStream_t st) {
  const bool aligned = p.K % TypeInfo<T>::VEC == 0;
  if (p.epi == EPI_OUT) return aligned ? skinny_rows<T, true, EPI_OUT>(p, st) : skinny_rows<T, false, EPI_OUT>(p, st);
  return aligned ? skinny_rows<T, true, EPI_LSE>(p, st) : skinny_rows<T, false, EPI_LSE>(p, st);
}

// A grid of one dimension holds 2^32 threads: many workgroups are dealt over
// two.
constexpr long GRID_X = 1 << 20;
inline dim3 grid_of(long wgs) {
  return wgs <= GRID_X ? dim3((unsigned)wgs) : dim3((unsigned)GRID_X, (unsigned)((wgs + GRID_X - 1) / GRID_X));
}
__device__ __forceinline__ long workgroup() { return (long)blockIdx.y * GRID_X + blockIdx.x; }

// ------------------------------------------------------------ operands
//
// Bound by memory (x of 4096 x 2048 bf16 without its padding rows: 7 us).
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(const T* __restrict__ in, T* __restrict__ out, long rows,
                                                   const T* __restrict__ in2, T* __restrict__ out2, long rows2, int cols,
                                                   long ldo, const int32_t* __restrict__ labels, int classes) {
  constexpr int VEC = TypeInfo<T>::VEC;
  const long cpr = ldo / VEC;
  const long i = workgroup() * 256 + threadIdx.x;
  if (i >= (rows + rows2) * cpr) return;
  long row = i / cpr;
  const long at = i - row * cpr;
  if (row >= rows) {
    row -= rows;
    in = in2;
    out = out2;
  }
  const int c = (int)at * VEC;
  union { uint4 u; T e[VEC]; } v;
  v.u = make_uint4(0, 0, 0, 0);
  if (!labels || label_ok(labels[row], classes)) {
    const T* p = in + row * cols + c;
    if (cols % VEC == 0) {
      v.u = *(const uint4*)p;
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        if (c + j < cols) v.e[j] = p[j];
    }
  }
  *(uint4*)(out + row * ldo + c) = v.u;
}

__global__ __launch_bounds__(256) void zero_kernel(uint16_t* p, size_t n) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) p[i] = 0;
}

// A workgroup: `rpw` rows of 256 columns, a thread 8 columns of every eighth row.
// Bound by memory (4000 x 4096 bf16, GELU, 98 MB: 21 us, 4.6 TB/s; with the two
// further terms, 164 MB, 31 us, 5.3), few rows by the latency of a
// thread's rows one after the other, so that a workgroup takes fewer of them.
template <typename T>
__global__ __launch_bounds__(256) void dact_kernel(int act, const T* __restrict__ dy, const T* __restrict__ z,
                                                   T* __restrict__ dz, bf16_t* __restrict__ more, float* __restrict__ colsum,
                                                   long rows, long rows_padded, int cols, long ldz, int rpw) {
  __shared__ float red[8][8 * 33];  // column 8 c + j at 33 j + c: no two lanes of a write in one bank
  const int tc = threadIdx.x & 31, tr = threadIdx.x >> 5;
  const int col = blockIdx.y * 256 + tc * 8;
  const long row0 = (long)blockIdx.x * rpw;
  const bool vec = cols % 8 == 0;
  float cs[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) cs[j] = 0.f;
  if (col < ldz) {
#pragma unroll 2
    for (int i = 0; i < rpw; i += 8) {
      const long row = row0 + i + tr;
      if (row >= rows_padded) break;
      float v[8], u[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = u[j] = 0.f;
      // the columns past a row's end (ldz may hold 64 more, and the last row has
      // no next one behind it) are written as zeros and never read
      if (row < rows && col < cols) {
        const long o = row * cols + col;
        if (vec) {  // a whole group of 8, or none
          load8<T>(dy + o, v);
          if (act) load8<T>(z + o, u);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (col + j < cols) {
              v[j] = elem_f(dy[o + j]);
              if (act) u[j] = elem_f(z[o + j]);
            }
        }
        // where ReLU passes nothing the gradient is zero, whatever dy holds
        if (act == ACT_RELU) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = u[j] > 0.f ? v[j] : 0.f;
        } else if (act) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] *= act_slope<T>(u[j], act);
        }
        if (!vec) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = col + j < cols ? v[j] : 0.f;
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) cs[j] += v[j];
      if (dz) store_terms<T>(dz, more, (size_t)(row * ldz + col), (size_t)(rows_padded * ldz), v);
    }
  }
  if (!colsum) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) red[tr][j * 33 + tc] = cs[j];
  __syncthreads();
  const int c = blockIdx.y * 256 + threadIdx.x;
  if (c >= cols || row0 >= rows) return;
  float s = 0.f;
#pragma unroll
  for (int r = 0; r < 8; ++r) s += red[r][(threadIdx.x & 7) * 33 + (threadIdx.x >> 3)];
  colsum[(long)blockIdx.x * cols + c] = s;
}

__global__ __launch_bounds__(256) void colsum_rows_kernel(const float* __restrict__ in, long ld, float* __restrict__ colsum,
                                                          long rows, int cols, const int32_t* __restrict__ labels,
                                                          int classes) {
  __shared__ float red[4][64];
  const int tc = threadIdx.x & 63, tr = threadIdx.x >> 6;
  const int col = blockIdx.y * 64 + tc;
  const long row0 = (long)blockIdx.x * COLSUM_ROWS;
  float s = 0.f;
  if (col < cols)
    for (int i = tr; i < COLSUM_ROWS && row0 + i < rows; i += 4)
      s += label_ok(labels[row0 + i], classes) ? in[(row0 + i) * ld + col] : 0.f;
  red[tr][tc] = s;
  __syncthreads();
  if (tr == 0 && col < cols) colsum[(long)blockIdx.x * cols + col] = red[0][tc] + red[1][tc] + red[2][tc] + red[3][tc];
}

__global__ __launch_bounds__(256) void column_sums_kernel(ColumnSums a) {
  __shared__ __align__(16) char lds[SUMS_LDS];
  column_sums(a, blockIdx.x, lds);
}

template <typename T>
__global__ __launch_bounds__(256) void round_rows_kernel(const float* __restrict__ in, T* __restrict__ out, long rows,
                                                         int cols, const int32_t* __restrict__ labels, int classes) {
  const long i = (workgroup() * 256 + threadIdx.x) * 4;
  const long n = rows * cols;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (i + j < n) store_out<T>(out + i + j, label_ok(labels[(i + j) / cols], classes) ? in[i + j] : 0.f);
}

// ---------------------------------------------------------------- loss rows
// (maximum, sum of exponentials relative to it) of two sets; an empty set's
// maximum is -inf and its sum 0.  NaN sums stay NaN.
__device__ __forceinline__ void merge(float& m, float& s, float m2, float s2) {
  const float mx = fmaxf(m, m2);
  const float base = mx == -INFINITY ? 0.f : mx;
  s = s * exp_fast(m - base) + s2 * exp_fast(m2 - base);
  m = mx;
}

// Over W threads (a wave, or a whole workgroup) that each hold a set.
template <int W> __device__ __forceinline__ void merge_all(float& m, float& s, float2* lds) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const float m2 = __shfl_xor(m, d), s2 = __shfl_xor(s, d);
    merge(m, s, m2, s2);
  }
  if constexpr (W > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = make_float2(m, s);
    __syncthreads();
    m = lds[0].x;
    s = lds[0].y;
#pragma unroll
    for (int i = 1; i < W / 64; ++i) merge(m, s, lds[i].x, lds[i].y);
  }
}

// logsumexp of a row from its groups' maxima and sums, W threads per row.  Bound
// by memory: 4096 rows of 1563 groups, 51 MB, 18 us.
template <int W>
__global__ __launch_bounds__(256) void lse_kernel(const float2* __restrict__ stats, int nstat, const float* __restrict__ zlab,
                                                  const int32_t* __restrict__ labels, int classes, long rows,
                                                  float2* __restrict__ lse, float* __restrict__ loss) {
  __shared__ float2 lds[4];
  const int t = threadIdx.x % W;
  const long row = workgroup() * (256 / W) + threadIdx.x / W;
  if (row >= rows) return;  // whole waves (W = 64), or no workgroup at all
  float m = -INFINITY, s = 0.f;
  const float2* p = stats + (size_t)row * nstat;
  for (int i = t; i < nstat; i += W) merge(m, s, p[i].x, p[i].y);
  merge_all<W>(m, s, lds);
  if (t == 0) {
    if (lse) lse[row] = row_lse(m, s);
    loss[1 + row] = label_ok(labels[row], classes) ? row_loss(m, s, zlab[row]) : 0.f;
  }
}

// One workgroup: the mean over the counted rows, in a fixed order, and what a
// counted row's gradient is multiplied with.
__global__ __launch_bounds__(1024) void loss_mean_kernel(const int32_t* __restrict__ labels, int classes, long rows,
                                                         float* __restrict__ loss, float* __restrict__ unit, float scale) {
  __shared__ double lds[16];
  double n = 0, s = 0;
  for (long r = threadIdx.x; r < rows; r += 1024) {
    const bool ok = label_ok(labels[r], classes);
    n += ok;
    if (ok) s += loss[1 + r];
  }
  n = block_sum(n, lds);
  s = block_sum(s, lds);
  if (threadIdx.x) return;
  loss[0] = n > 0 ? (float)(s / n) : 0.f;
  if (unit) unit[0] = n > 0 ? (float)(scale / n) : 0.f;
}

// W threads per row of kept logits, given as the partial sums of their product
// (S of them, without the bias).  The first pass adds them up, leaves the logit
// in the first one's place and takes the maximum and sum as it goes; the second
// reads the logits back (from the thread's own stores) and leaves the unrounded
// dlogits there for the column sums.  The row of x goes along, cleaned.  Bound by
// latency where rows are few (256 x 1000 bf16 9 us, 333 x 5003 fp32 13 us).
template <typename T, int W>
__global__ __launch_bounds__(W > 256 ? W : 256) void loss_rows_kernel(LossRows a) {
  __shared__ float2 lds[16];
  __shared__ float zl[4];
  constexpr int WG = W > 256 ? W : 256;
  const int t = threadIdx.x % W, in_wg = threadIdx.x / W;
  const long row = (long)blockIdx.x * (WG / W) + in_wg;
  if (a.unit && blockIdx.x == 0) {  // (up to FINISH_ROWS rows)
    __shared__ double cnt[16];
    double n = 0;
    for (long r = threadIdx.x; r < a.rows; r += WG) n += label_ok(a.labels[r], a.classes);
    n = block_sum(n, cnt);
    if (threadIdx.x == 0) a.unit[0] = n > 0 ? (float)(a.scale / n) : 0.f;
  }
  if (row >= a.rows_padded) return;
  const int lab = row < a.rows ? a.labels[row] : -1;
  const bool live = label_ok(lab, a.classes);
  if (a.xc && row < a.rows) {
    constexpr int VEC = TypeInfo<T>::VEC;
    const T* xr = (const T*)a.x + row * a.in;
    T* o = (T*)a.xc + row * a.ldx;
    for (int c = t * VEC; c < a.ldx; c += W * VEC) {
      union { uint4 u; T e[VEC]; } v;
      v.u = make_uint4(0, 0, 0, 0);
      if (live) {
        if (a.in % VEC == 0) {
          v.u = *(const uint4*)(xr + c);
        } else {
#pragma unroll
          for (int j = 0; j < VEC; ++j)
            if (c + j < a.in) v.e[j] = xr[c + j];
        }
      }
      *(uint4*)(o + c) = v.u;
    }
  }
  float* zr = a.z + (size_t)(row < a.rows ? row : 0) * a.ldz;
  const size_t step = (size_t)a.rows * a.ldz;
  float2 lse = make_float2(0.f, 0.f);
  float m = -INFINITY, s = 0.f;
  if (live) {  // the same for all threads of a row
    constexpr int U = 4;
    for (int c0 = t; c0 < a.classes; c0 += U * W) {
      float v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = c0 + u * W < a.classes ? zr[c0 + u * W] : -INFINITY;
      for (int p = 1; p < a.splits; ++p) {
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] += c0 + u * W < a.classes ? zr[p * step + c0 + u * W] : 0.f;
      }
      float mx = m;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + u * W;
        if (c < a.classes) {
          if (a.bias) v[u] += a.bias[c];
          zr[c] = v[u];
          if (c == lab) zl[in_wg] = v[u];
        }
        mx = fmaxf(mx, v[u]);
      }
      const float base = mx == -INFINITY ? 0.f : mx;
      s *= exp_fast(m - base);
#pragma unroll
      for (int u = 0; u < U; ++u) s += exp_fast(v[u] - base);
      m = mx;
    }
    merge_all<W>(m, s, lds);
    lse = row_lse(m, s);
  }
  if constexpr (W > 64) __syncthreads();  // the label's logit
  __builtin_amdgcn_wave_barrier();
  if (t == 0 && row < a.rows) a.loss[1 + row] = live ? row_loss(m, s, zl[in_wg]) : 0.f;
  if (!a.dz) return;
  for (long c = t; c < a.ldd; c += W) {
    float v = 0.f;
    if (live && c < a.classes) v = row_prob(zr[c], lse) - (c == lab ? 1.f : 0.f);
    store_out<T>((T*)a.dz + row * a.ldd + c, v);
    if (sizeof(T) == 2 && a.more) {
      float left = v;
      for (int i = 0; i < TERMS - 1; ++i) {
        left -= bf16_to_f32(f32_to_bf16(left));
        ((bf16_t*)a.more)[(i * a.rows_padded + row) * a.ldd + c] = f32_to_bf16(left);
      }
    }
    if (a.keep_dz && row < a.rows && c < a.classes) zr[c] = v;
  }
}

// The same for many classes, LOSS_PART of them per workgroup (x: of the row,
// y: part), in two launches: the first adds the partial sums up, leaves the
// logits and the part's maximum and sum, and cleans x; the second merges the
// parts' and does the rest.
__global__ __launch_bounds__(256) void loss_parts_kernel(LossRows a, float2* __restrict__ stats, int parts) {
  __shared__ float2 lds[4];
  const long row = blockIdx.x;
  if (a.unit && blockIdx.x == 0 && blockIdx.y == 0) {
    __shared__ double cnt[4];
    double n = 0;
    for (long r = threadIdx.x; r < a.rows; r += 256) n += label_ok(a.labels[r], a.classes);
    n = block_sum(n, cnt);
    if (threadIdx.x == 0) a.unit[0] = n > 0 ? (float)(a.scale / n) : 0.f;
  }
  if (!label_ok(a.labels[row], a.classes)) return;
  constexpr int U = 4;
  float* zr = a.z + (size_t)row * a.ldz;
  const size_t step = (size_t)a.rows * a.ldz;
  const int end = min(a.classes, (int)(blockIdx.y + 1) * LOSS_PART);
  float m = -INFINITY, s = 0.f;
  for (int c0 = blockIdx.y * LOSS_PART + threadIdx.x; c0 < end; c0 += U * 256) {
    float v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = c0 + u * 256 < end ? zr[c0 + u * 256] : -INFINITY;
    for (int p = 1; p < a.splits; ++p) {
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] += c0 + u * 256 < end ? zr[p * step + c0 + u * 256] : 0.f;
    }
    float mx = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * 256;
      if (c < end) {
        if (a.bias) v[u] += a.bias[c];
        zr[c] = v[u];
      }
      mx = fmaxf(mx, v[u]);
    }
    const float base = mx == -INFINITY ? 0.f : mx;
    s *= exp_fast(m - base);
#pragma unroll
    for (int u = 0; u < U; ++u) s += exp_fast(v[u] - base);
    m = mx;
  }
  merge_all<256>(m, s, lds);
  if (threadIdx.x == 0) stats[row * parts + blockIdx.y] = make_float2(m, s);
}

template <typename T>
__global__ __launch_bounds__(256) void loss_parts_end_kernel(LossRows a, const float2* __restrict__ stats, int parts) {
  const long row = blockIdx.x;
  const int lab = row < a.rows ? a.labels[row] : -1;
  const bool live = label_ok(lab, a.classes);
  float* zr = a.z + (size_t)(row < a.rows ? row : 0) * a.ldz;
  float2 lse = make_float2(0.f, 0.f);
  float m = -INFINITY, s = 0.f;
  if (live) {
    for (int i = threadIdx.x & 63; i < parts; i += 64) merge(m, s, stats[row * parts + i].x, stats[row * parts + i].y);
    merge_all<64>(m, s, nullptr);
    lse = row_lse(m, s);
  }
  const int lo = blockIdx.y * LOSS_PART, hi = (int)min((long)lo + LOSS_PART, a.dz ? a.ldd : (long)a.classes);
  // the part that holds the label, or the first one of a padding row
  if (row < a.rows && threadIdx.x == 0 && (live ? lab >= lo && lab < lo + LOSS_PART : blockIdx.y == 0))
    a.loss[1 + row] = live ? row_loss(m, s, zr[lab]) : 0.f;
  if (!a.dz) return;
  __syncthreads();  // the label's logit is read before its place is written
  if (a.xc && row < a.rows) {
    constexpr int VEC = TypeInfo<T>::VEC;
    const T* xr = (const T*)a.x + row * a.in;
    T* o = (T*)a.xc + row * a.ldx;
    for (long c = ((long)blockIdx.y * 256 + threadIdx.x) * VEC; c < a.ldx; c += (long)gridDim.y * 256 * VEC) {
      union { uint4 u; T e[VEC]; } v;
      v.u = make_uint4(0, 0, 0, 0);
      if (live) {
#pragma unroll
        for (int j = 0; j < VEC; ++j)
          if (c + j < a.in) v.e[j] = xr[c + j];
      }
      *(uint4*)(o + c) = v.u;
    }
  }
  for (int c = lo + threadIdx.x; c < hi; c += 256) {
    float v = 0.f;
    if (live && c < a.classes) v = row_prob(zr[c], lse) - (c == lab ? 1.f : 0.f);
    store_out<T>((T*)a.dz + row * a.ldd + c, v);
    if (sizeof(T) == 2 && a.more) {
      float left = v;
      for (int i = 0; i < TERMS - 1; ++i) {
        left -= bf16_to_f32(f32_to_bf16(left));
        ((bf16_t*)a.more)[(i * a.rows_padded + row) * a.ldd + c] = f32_to_bf16(left);
      }
    }
    if (a.keep_dz && row < a.rows && c < a.classes) zr[c] = v;
  }
}

__global__ __launch_bounds__(256) void loss_finish_kernel(LossFinish f) {
  __shared__ __align__(16) char lds[FINISH_LDS];
  loss_finish(f, blockIdx.x, lds);
}

// One or a few rows of many column groups: the loss of each, and the mean.
__global__ __launch_bounds__(1024) void lse_finish_kernel(const float2* __restrict__ stats, int nstat,
                                                          const float* __restrict__ zlab, const int32_t* __restrict__ labels,
                                                          int classes, int rows, float* __restrict__ loss) {
  __shared__ float2 lds[16];
  double sum = 0;
  int n = 0;
  for (int row = 0; row < rows; ++row) {
    float m = -INFINITY, s = 0.f;
    for (int i = threadIdx.x; i < nstat; i += 1024) {
      const float2 p = stats[(size_t)row * nstat + i];
      merge(m, s, p.x, p.y);
    }
    merge_all<1024>(m, s, lds);
    __syncthreads();
    const bool ok = label_ok(labels[row], classes);
    const float l = ok ? row_loss(m, s, zlab[row]) : 0.f;
    if (threadIdx.x == 0) loss[1 + row] = l;
    sum += l;
    n += ok;
  }
  if (threadIdx.x == 0) loss[0] = n ? (float)(sum / n) : 0.f;
}

// The same, a wave per row: few rows of few column groups.
__global__ __launch_bounds__(1024) void lse_finish_rows_kernel(const float2* __restrict__ stats, int nstat,
                                                               const float* __restrict__ zlab,
                                                               const int32_t* __restrict__ labels, int classes, int rows,
                                                               float* __restrict__ loss) {
  __shared__ double lds[16];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  double sum = 0, n = 0;
  for (int row = wave; row < rows; row += 16) {
    float m = -INFINITY, s = 0.f;
    for (int i = lane; i < nstat; i += 64) {
      const float2 p = stats[(size_t)row * nstat + i];
      merge(m, s, p.x, p.y);
    }
    merge_all<64>(m, s, nullptr);
    if (lane) continue;
    const bool ok = label_ok(labels[row], classes);
    const float l = ok ? row_loss(m, s, zlab[row]) : 0.f;
    loss[1 + row] = l;
    sum += l;
    n += ok;
  }
  n = block_sum(n, lds);
  sum = block_sum(sum, lds);
  if (threadIdx.x == 0) loss[0] = n > 0 ? (float)(sum / n) : 0.f;
}

}  // namespace

hipError_t launch_zero(void* p, size_t bytes, hipStream_t st) {
  TraceScope ts("zero_kernel", st, (double)bytes, WORK_BYTE);
  const size_t n = bytes / 2, wgs = (n + 255) / 256;
  hipLaunchKernelGGL(zero_kernel, dim3((unsigned)(wgs < 4096 ? wgs : 4096)), dim3(256), 0, st, (uint16_t*)p, n);
  return hipGetLastError();
}

hipError_t launch_skinny(const Product& p, hipStream_t st) { return p.dt == BF16 ? skinny_t<bf16_t>(p, st) : skinny_t<float>(p, st); }

static hipError_t pack(int dt, const void* in, void* out, long rows, const void* in2, void* out2, long rows2, int cols,
                       long ldo, const int32_t* labels, int classes, hipStream_t st) {
  TraceScope ts("pack_kernel", st, (double)(rows + rows2) * (cols + ldo) * dt_size(dt), WORK_BYTE);
  const long chunks = (rows + rows2) * (ldo / (dt == BF16 ? 8 : 4));
  const dim3 grid = grid_of((chunks + 255) / 256);
  if (dt == BF16)
    hipLaunchKernelGGL(pack_kernel<bf16_t>, grid, dim3(256), 0, st, (const bf16_t*)in, (bf16_t*)out, rows, (const bf16_t*)in2,
                       (bf16_t*)out2, rows2, cols, ldo, labels, classes);
  else
    hipLaunchKernelGGL(pack_kernel<float>, grid, dim3(256), 0, st, (const float*)in, (float*)out, rows, (const float*)in2,
                       (float*)out2, rows2, cols, ldo, labels, classes);
  return hipGetLastError();
}

hipError_t launch_pack(int dt, const void* in, void* out, long rows, int cols, long ldo, const int32_t* labels, int classes,
                       hipStream_t st) {
  return pack(dt, in, out, rows, nullptr, nullptr, 0, cols, ldo, labels, classes, st);
}

hipError_t launch_pack2(int dt, const void* in, void* out, long rows, const void* in2, void* out2, long rows2, int cols,
                        long ldo, hipStream_t st) {
  return pack(dt, in, out, rows, in2, out2, rows2, cols, ldo, nullptr, 0, st);
}

// Halved until there are two workgroups per CU (256 x 4096 bf16, GELU: 64
// workgroups of 64 rows took 9.6 us).
int dact_rows(long rows, int cols) {
  int rpw = COLSUM_ROWS;
  while (rpw > 8 && (rows + rpw - 1) / rpw * ((cols + 255) / 256) < 512) rpw /= 2;
  return rpw;
}

hipError_t launch_dact(int dt, int act, const void* dy, const void* z, void* dz, void* more, float* colsum, long rows,
                       long rows_padded, int cols, long ldz, hipStream_t st) {
  const int rpw = dact_rows(rows, cols);
  const dim3 grid((unsigned)((rows_padded + rpw - 1) / rpw), (unsigned)((ldz + 255) / 256));
  TraceScope ts("dact_kernel", st, (double)rows * cols * dt_size(dt) * (1 + (act != 0) + (dz != nullptr) + (more ? TERMS - 1 : 0)),
                WORK_BYTE);
  if (dt == BF16)
    hipLaunchKernelGGL(dact_kernel<bf16_t>, grid, dim3(256), 0, st, act, (const bf16_t*)dy, (const bf16_t*)z, (bf16_t*)dz,
                       (bf16_t*)more, colsum, rows, rows_padded, cols, ldz, rpw);
  else
    hipLaunchKernelGGL(dact_kernel<float>, grid, dim3(256), 0, st, act, (const float*)dy, (const float*)z, (float*)dz,
                       (bf16_t*)nullptr, colsum, rows, rows_padded, cols, ldz, rpw);
  return hipGetLastError();
}

hipError_t launch_column_sums(const ColumnSums& s, hipStream_t st) {
  TraceScope ts("column_sums_kernel", st, (double)dt_size(s.dt) * s.rows * s.cols, WORK_BYTE);
  hipLaunchKernelGGL(column_sums_kernel, dim3(sums_wgs(s)), dim3(256), 0, st, s);
  return hipGetLastError();
}

hipError_t launch_colsum_rows(const float* dzf, long ld, float* colsum, long rows, int cols, const int32_t* labels,
                              int classes, hipStream_t st) {
  TraceScope ts("colsum_rows_kernel", st, 4.0 * rows * cols, WORK_BYTE);
  const dim3 grid((unsigned)((rows + COLSUM_ROWS - 1) / COLSUM_ROWS), (unsigned)((cols + 63) / 64));
  hipLaunchKernelGGL(colsum_rows_kernel, grid, dim3(256), 0, st, dzf, ld, colsum, rows, cols, labels, classes);
  return hipGetLastError();
}

hipError_t launch_round_rows(int dt, const float* in, void* out, long rows, int cols, const int32_t* labels, int classes,
                             hipStream_t st) {
  TraceScope ts("round_rows_kernel", st, (double)rows * cols * (4 + dt_size(dt)), WORK_BYTE);
  const dim3 grid = grid_of((rows * cols + 1023) / 1024);
  if (dt == BF16)
    hipLaunchKernelGGL(round_rows_kernel<bf16_t>, grid, dim3(256), 0, st, in, (bf16_t*)out, rows, cols, labels, classes);
  else
    hipLaunchKernelGGL(round_rows_kernel<float>, grid, dim3(256), 0, st, in, (float*)out, rows, cols, labels, classes);
  return hipGetLastError();
}

hipError_t launch_lse(const float2* stats, int nstat, const float* zlab, const int32_t* labels, int classes, long rows,
                      float2* lse, float* loss, hipStream_t st) {
  TraceScope ts("lse_kernel", st, 8.0 * rows * nstat, WORK_BYTE);
  // a wave per row, or, where rows are few, a workgroup per row (loss alone, bf16,
  // 64 inputs, wave / workgroup: 300 x 100000 45 / 39 us, 600 x 100000 63 / 57,
  // 900 x 32000 41 / 39, 1500 x 100000 126 / 120, 3000 x 32000 101 / 102)
  if (rows >= 1024)
    hipLaunchKernelGGL(lse_kernel<64>, grid_of((rows + 3) / 4), dim3(256), 0, st, stats, nstat, zlab, labels, classes,
                       rows, lse, loss);
  else
    hipLaunchKernelGGL(lse_kernel<256>, dim3((unsigned)rows), dim3(256), 0, st, stats, nstat, zlab, labels, classes, rows, lse,
                       loss);
  return hipGetLastError();
}

hipError_t launch_loss_mean(const int32_t* labels, int classes, long rows, float* loss, float* unit, float scale,
                            hipStream_t st) {
  TraceScope ts("loss_mean_kernel", st, 8.0 * rows, WORK_BYTE);
  hipLaunchKernelGGL(loss_mean_kernel, dim3(1), dim3(1024), 0, st, labels, classes, rows, loss, unit, scale);
  return hipGetLastError();
}

hipError_t launch_loss_rows(int dt, const LossRows& a, hipStream_t st) {
  // One row per workgroup leaves the chip empty where rows are few and long:
  // 64 rows of 50000 classes took 122 us.
  if (a.stats) {
    const int parts = loss_parts(a.classes);
    {
      TraceScope ts("loss_parts_kernel", st, 4.0 * a.rows * a.classes * (a.splits + 1), WORK_BYTE);
      hipLaunchKernelGGL(loss_parts_kernel, dim3((unsigned)a.rows, parts), dim3(256), 0, st, a, a.stats, parts);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    TraceScope ts("loss_parts_end_kernel", st, (double)a.rows * a.classes * (8 + dt_size(dt)), WORK_BYTE);
    const dim3 grid((unsigned)a.rows_padded, (unsigned)(a.dz ? (a.ldd + LOSS_PART - 1) / LOSS_PART : parts));
    if (dt == BF16)
      hipLaunchKernelGGL(loss_parts_end_kernel<bf16_t>, grid, dim3(256), 0, st, a, a.stats, parts);
    else
      hipLaunchKernelGGL(loss_parts_end_kernel<float>, grid, dim3(256), 0, st, a, a.stats, parts);
    return hipGetLastError();
  }
  TraceScope ts("loss_rows_kernel", st, (double)a.rows * a.classes * (8 + dt_size(dt)), WORK_BYTE);
  // a wave per row of few classes, else a workgroup, of 1024 threads where rows
  // are too few for the chip to fill otherwise
  const int w = a.classes <= 256 ? 64 : a.classes > 2048 && a.rows < 1024 ? 1024 : 256;
  const dim3 grid((unsigned)(w == 64 ? (a.rows_padded + 3) / 4 : a.rows_padded)), wg(w == 64 ? 256 : w);
#define SINGA_ROWS(T)                                                            \
  if (w == 64)                                                                   \
    hipLaunchKernelGGL((loss_rows_kernel<T, 64>), grid, wg, 0, st, a);           \
  else if (w == 256)                                                             \
    hipLaunchKernelGGL((loss_rows_kernel<T, 256>), grid, wg, 0, st, a);          \
  else                                                                           \
    hipLaunchKernelGGL((loss_rows_kernel<T, 1024>), grid, wg, 0, st, a)
  if (dt == BF16) {
    SINGA_ROWS(bf16_t);
  } else {
    SINGA_ROWS(float);
  }
#undef SINGA_ROWS
  return hipGetLastError();
}

hipError_t launch_loss_finish(const LossFinish& f, hipStream_t st) {
  TraceScope ts("loss_finish_kernel", st, f.db ? 4.0 * f.rows * f.classes : 8.0 * f.rows, WORK_BYTE);
  hipLaunchKernelGGL(loss_finish_kernel, dim3(finish_wgs(f)), dim3(256), 0, st, f);
  return hipGetLastError();
}

hipError_t launch_lse_finish(const float2* stats, int nstat, const float* zlab, const int32_t* labels, int classes, int rows,
                             float* loss, hipStream_t st) {
  TraceScope ts("lse_finish_kernel", st, 8.0 * rows * nstat, WORK_BYTE);
  if (rows <= LSE_FINISH_ROWS)
    hipLaunchKernelGGL(lse_finish_kernel, dim3(1), dim3(1024), 0, st, stats, nstat, zlab, labels, classes, rows, loss);
  else
    hipLaunchKernelGGL(lse_finish_rows_kernel, dim3(1), dim3(1024), 0, st, stats, nstat, zlab, labels, classes, rows, loss);
  return hipGetLastError();
}

}  // namespace singa
