// The contraction kernel for x W^T of 8-bit integers, the lower tiles (a file of its own only to compile in parallel).
#include "gemm_ring.h"

#define I8_SHAPES(X) X(3, 128, 256, 3) X(6, 128, 192, 3) X(8, 128, 128, 4) X(9, 64, 128, 4) X(10, 128, 64, 4) X(11, 64, 64, 4)
#define I8_INST(I, BM, BN, NS) template __global__ void gemm_bf16_ring_kernel<BM, BN, NS, false, false, false, GEMM_EPIS_I8, false, true>(const RingGrid, const GemmDesc);
I8_SHAPES(I8_INST)

hipError_t gemm_ring_launch_i8_small(ecospa_ctx* ctx, const GemmDesc& d, int shape, int k_chunk) {
#define I8_CASE(I, BM, BN, NS) if (shape == I) return ring_launch_shape<BM, BN, NS, false, false, false, GEMM_EPIS_I8, false, true>(ctx, d, k_chunk);
  I8_SHAPES(I8_CASE)
  return hipErrorInvalidValue;
}
