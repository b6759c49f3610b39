// dense_f32.hip -- the dense products of fp32 operands (dense_gemm.h), and the
// choice between the two types.
#include "dense_gemm.h"

namespace singa {

hipError_t launch_product_bf16(const Product& p, float* partial, hipStream_t st);
hipError_t launch_pair_bf16(const Product& dx, const Product& dw, const ColumnSums* sums, const LossFinish* finish,
                            float* partial, hipStream_t st);

size_t product_partial_bytes(int dt, int M, int N, int K, int epi) {
  return partial_bytes_of(plan_product(dt, M, N, K, epi), M, N);
}

size_t pair_partial_bytes(int dt, int Ma, int Na, int Ka, int Mb, int Nb, int Kb) {
  const PairPlan p = plan_pair(dt, Ma, Na, Ka, Mb, Nb, Kb);
  return pair_pays(dt, p, Ma, Na, Ka, Mb, Nb, Kb) ? partial_bytes_of(p.a, Ma, Na) + partial_bytes_of(p.b, Mb, Nb) : 0;
}

bool product_skinny(int dt, int M, int N, int K, bool copied) { return skinny_pays(dt, M, N, K, copied); }

int product_splits(int dt, int M, int N, int K) { return plan_product(dt, M, N, K, EPI_OUT).splits; }

hipError_t launch_product(const Product& p, float* partial, hipStream_t st) {
  return p.dt == BF16 ? launch_product_bf16(p, partial, st) : launch_product_t<float>(p, partial, st);
}

hipError_t launch_pair(const Product& dx, const Product& dw, const ColumnSums* sums, const LossFinish* finish, float* partial,
                       hipStream_t st) {
  return dx.dt == BF16 ? launch_pair_bf16(dx, dw, sums, finish, partial, st)
                       : launch_pair_t<float>(dx, dw, sums, finish, partial, st);
}

}  // namespace singa
