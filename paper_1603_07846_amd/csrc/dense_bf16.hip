// dense_bf16.hip -- the dense products of bf16 operands (dense_gemm.h).
#include "dense_gemm.h"

namespace singa {

hipError_t launch_product_bf16(const Product& p, float* partial, hipStream_t st) {
  return launch_product_t<bf16_t>(p, partial, st);
}

hipError_t launch_pair_bf16(const Product& dx, const Product& dw, const ColumnSums* sums, const LossFinish* finish,
                            float* partial, hipStream_t st) {
  return launch_pair_t<bf16_t>(dx, dw, sums, finish, partial, st);
}

}  // namespace singa
