// gradnorm.hip -- the global norm over many gradient tensors, and clipping.
//
// Bound by memory: the norm reads every gradient once, clipping reads and
// writes it once more (the scale has to be known first); 62 M fp32 values: the
// norm 48 us, 5.2 TB/s; 120 M bf16 values: scaling 77 us, 6.2 TB/s.  The tensors' list
// travels in the kernel arguments, LIST tensors a launch, so that a captured
// call holds its own copy and nothing is copied to the device.  Each
// workgroup sums the squares of one piece of one tensor in fp64 (the card's
// fp64 rate is far above what the loads deliver, and no square overflows or
// vanishes) into its own slot; one workgroup adds the slots in order, or, when
// clipping has few of them, every workgroup that scales does.
#include "conv_common.h"
#include "gradnorm.h"

namespace singa {

namespace {

typedef uint32_t u4v __attribute__((ext_vector_type(4)));

// One record per tensor, of a size that keeps every field's address aligned
// whatever the index.  (With an array of bytes beside arrays of pointers the
// compiler took base + index as the common address of both and split the
// pointers' offset into index + 7 index; scalar loads drop the low bits of
// each part, and wrong pointers came back.)
struct Item {
  const void* p;
  void* out;
  uint64_t n;
  uint32_t first;  // the tensor's first workgroup of this launch
  uint32_t dt;
};
static_assert(sizeof(Item) == 32, "aligned records");

struct List {
  Item t[NORM_LIST];
  int count;
  uint32_t slot0;
  uint64_t piece;  // elements per workgroup
};

// The tensor and the range of elements of this workgroup.
__device__ __forceinline__ int find(const List& l, uint32_t b, uint64_t& lo, uint64_t& hi) {
  int i = 0;
  for (int d = 64; d; d >>= 1)
    if (i + d < l.count && l.t[i + d].first <= b) i += d;
  lo = (uint64_t)(b - l.t[i].first) * l.piece;
  hi = lo + l.piece < l.t[i].n ? lo + l.piece : l.t[i].n;
  return i;
}

__device__ __forceinline__ void sq(double& s, float v) { s = fma((double)v, (double)v, s); }
__device__ __forceinline__ float lo_bf(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_bf(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

template <typename T> __device__ __forceinline__ void sq16(double& s0, double& s1, const u4v& w) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (sizeof(T) == 4) {
      sq(j & 1 ? s1 : s0, __uint_as_float(w[j]));
    } else {
      sq(s0, lo_bf(w[j]));
      sq(s1, hi_bf(w[j]));
    }
  }
}

constexpr int U = 4;  // 16-byte loads in flight per thread

// Sum of squares of p[0 .. n): elements up to the first 16-byte boundary and
// from the last one on one by one, 16-byte loads between them.
template <typename T> __device__ __forceinline__ double piece_sq(const T* p, uint64_t n) {
  constexpr int VEC = 16 / (int)sizeof(T);
  const int t = threadIdx.x;
  uint64_t head = (16 - ((uintptr_t)p & 15)) / sizeof(T) % VEC;
  if (head > n) head = n;
  double s0 = 0, s1 = 0;
  if ((uint64_t)t < head) sq(s0, elem_f(p[t]));
  const u4v* v = (const u4v*)(p + head);
  const uint64_t nv = (n - head) / VEC;
  uint64_t i = t;
  for (; i + (U - 1) * 256 < nv; i += U * 256) {
    u4v w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = v[i + u * 256];
#pragma unroll
    for (int u = 0; u < U; ++u) sq16<T>(s0, s1, w[u]);
  }
  for (; i < nv; i += 256) sq16<T>(s0, s1, v[i]);
  const uint64_t done = head + nv * VEC;
  if (done + t < n) sq(s1, elem_f(p[done + t]));
  return s0 + s1;
}

__device__ __forceinline__ double wg_sum(double s, double* lds, int waves) {
#pragma unroll
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0;
  for (int i = 0; i < waves; ++i) s += lds[i];
  return s;
}

__global__ __launch_bounds__(256) void grad_sq_kernel(List l, double* __restrict__ slots) {
  __shared__ double lds[4];
  uint64_t lo, hi;
  const int i = find(l, blockIdx.x, lo, hi);
  const void* p = l.t[i].p;
  const double s = l.t[i].dt == BF16 ? piece_sq((const bf16_t*)p + lo, hi - lo) : piece_sq((const float*)p + lo, hi - lo);
  const double all = wg_sum(s, lds, 4);
  if (threadIdx.x == 0) slots[l.slot0 + blockIdx.x] = all;
}

// The norm and the scale from the slots, the same in every thread and for
// every number of threads a multiple of 256 (thread t adds slots t, t + 256, ...
// of the first 256 threads).
__device__ __forceinline__ float2 norm_of(const double* __restrict__ slots, uint32_t n, float max_norm, double* lds) {
  double s = 0;
  if (threadIdx.x < 256)
    for (uint32_t i = threadIdx.x; i < n; i += 256) s += slots[i];
  const double norm = sqrt(wg_sum(s, lds, (int)blockDim.x / 64));
  // a norm that is not finite compares false, or is excluded
  const bool over = norm > (double)max_norm && norm <= 1.7976931348623157e308;
  return make_float2((float)norm, over ? (float)((double)max_norm / norm) : 1.f);
}

__global__ __launch_bounds__(256) void grad_norm_kernel(const double* __restrict__ slots, uint32_t n, float max_norm,
                                                        float* __restrict__ stat) {
  __shared__ double lds[4];
  const float2 r = norm_of(slots, n, max_norm, lds);
  if (threadIdx.x) return;
  stat[0] = r.x;
  stat[1] = r.y;
}

template <typename T> __device__ __forceinline__ void piece_scale(const T* p, T* o, uint64_t n, float s) {
  constexpr int VEC = 16 / (int)sizeof(T);
  const int t = threadIdx.x;
  uint64_t head = (16 - ((uintptr_t)p & 15)) / sizeof(T) % VEC;
  if (head > n || (((uintptr_t)p ^ (uintptr_t)o) & 15)) head = n;  // starts that differ: element by element
  for (uint64_t i = t; i < head; i += 256) store_out<T>(o + i, elem_f(p[i]) * s);
  const u4v* v = (const u4v*)(p + head);
  u4v* q = (u4v*)(o + head);
  const uint64_t nv = (n - head) / VEC;
  auto scaled = [&](u4v w) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (sizeof(T) == 4)
        w[j] = __float_as_uint(__uint_as_float(w[j]) * s);
      else
        w[j] = f32x2_to_bf16x2(lo_bf(w[j]) * s, hi_bf(w[j]) * s);
    }
    return w;
  };
  uint64_t i = t;
  for (; i + (U - 1) * 256 < nv; i += U * 256) {
    u4v w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = __builtin_nontemporal_load(v + i + u * 256);
#pragma unroll
    for (int u = 0; u < U; ++u) __builtin_nontemporal_store(scaled(w[u]), q + i + u * 256);
  }
  for (; i < nv; i += 256) q[i] = scaled(v[i]);
  for (uint64_t j = head + nv * VEC + t; j < n; j += 256) store_out<T>(o + j, elem_f(p[j]) * s);
}

// n: number of slots to add here (0: stat is written already).  The first
// workgroup of the first launch writes stat then.
__global__ __launch_bounds__(256) void grad_scale_kernel(List l, float* __restrict__ stat, const double* __restrict__ slots,
                                                         uint32_t n, float max_norm) {
  __shared__ double lds[4];
  uint64_t lo, hi;
  const int i = find(l, blockIdx.x, lo, hi);
  float s;
  if (n) {
    const float2 r = norm_of(slots, n, max_norm, lds);
    s = r.y;
    if (l.slot0 + blockIdx.x + threadIdx.x == 0) {
      stat[0] = r.x;
      stat[1] = r.y;
    }
  } else {
    s = stat[1];
  }
  const void* p = l.t[i].p;
  void* o = l.t[i].out;
  if (s == 1.f && p == o) return;
  if (l.t[i].dt == BF16)
    piece_scale((const bf16_t*)p + lo, (bf16_t*)o + lo, hi - lo, s);
  else
    piece_scale((const float*)p + lo, (float*)o + lo, hi - lo, s);
}

}  // namespace

hipError_t launch_grad_norm(int count, const int* dt, const void* const* grads, void* const* outs, const size_t* sizes,
                            float max_norm, float* stat, double* slots, hipStream_t st) {
  uint64_t total = 0;
  double bytes = 0;
  for (int i = 0; i < count; ++i) total += sizes[i], bytes += (double)sizes[i] * dt_size(dt[i]);
  // at least 16,384 elements a workgroup, and at most NORM_PIECES whole pieces
  uint64_t piece = (total + NORM_PIECES - 1) / NORM_PIECES;
  piece = piece < 16384 ? 16384 : (piece + 8191) / 8192 * 8192;
  uint32_t slots_used = 0;
  bool sum_here = false;
  for (int pass = 0; pass < (outs ? 2 : 1); ++pass) {
    uint32_t slot = 0;
    for (int at = 0; at < count;) {
      List l{};
      l.slot0 = slot;
      l.piece = piece;
      uint32_t wgs = 0;
      for (; at < count && l.count < NORM_LIST; ++at) {
        if (!sizes[at]) continue;
        l.t[l.count++] = Item{grads[at], outs ? outs[at] : nullptr, sizes[at], wgs, (uint32_t)dt[at]};
        wgs += (uint32_t)((sizes[at] + piece - 1) / piece);
      }
      if (!l.count) break;
      slot += wgs;
      if (pass == 0) {
        TraceScope ts("grad_sq_kernel", st, bytes, WORK_BYTE);
        hipLaunchKernelGGL(grad_sq_kernel, dim3(wgs), dim3(256), 0, st, l, slots);
      } else {
        TraceScope ts("grad_scale_kernel", st, 2 * bytes, WORK_BYTE);
        hipLaunchKernelGGL(grad_scale_kernel, dim3(wgs), dim3(256), 0, st, l, stat, slots, sum_here ? slots_used : 0, max_norm);
      }
      bytes = 0;  // the trace counts the whole list at its first launch
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    if (pass) break;
    slots_used = slot;
    // A launch costs about 3 us; 512 slots are 4 KB that each workgroup reads
    // from a cache in well under 1.
    sum_here = outs && slots_used && slots_used <= 512;
    for (int i = 0; i < count; ++i) bytes += (double)sizes[i] * dt_size(dt[i]);
    if (sum_here) continue;
    TraceScope ts("grad_norm_kernel", st, 8.0 * slots_used, WORK_BYTE);
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(256), 0, st, slots, slots_used, max_norm, stat);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace singa
