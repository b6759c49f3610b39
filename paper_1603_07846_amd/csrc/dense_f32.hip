// dense_f32.hip -- the dense products of fp32 operands (dense_gemm.h), and the
// choice between the two types.
#include "dense_gemm.h"

namespace singa {

hipError_t launch_product_bf16(const Product& p, float* partial, hipStream_t st);

size_t product_partial_bytes(int dt, int M, int N, int K, int epi) {
  const Plan p = plan_product(dt, M, N, K, epi);
  return p.splits > 1 ? (size_t)p.splits * M * (((size_t)N + 7) / 8 * 8) * 4 : 0;
}

int product_splits(int dt, int M, int N, int K) { return plan_product(dt, M, N, K, EPI_OUT).splits; }

hipError_t launch_product(const Product& p, float* partial, hipStream_t st) {
  return p.dt == BF16 ? launch_product_bf16(p, partial, st) : launch_product_t<float>(p, partial, st);
}

}  // namespace singa
