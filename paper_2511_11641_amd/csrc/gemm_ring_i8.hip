// The contraction kernel for x W^T of 8-bit integers, 256- and 192-row tiles.
#include "gemm_ring.h"

#define I8_SHAPES(X) X(0, 256, 256, 2) X(1, 192, 256, 2) X(2, 256, 192, 2) X(4, 256, 128, 3) X(5, 192, 192, 3) X(7, 192, 128, 3)
#define I8_INST(I, BM, BN, NS) template __global__ void gemm_bf16_ring_kernel<BM, BN, NS, false, false, false, GEMM_EPIS_I8, false, true>(const RingGrid, const GemmDesc);
I8_SHAPES(I8_INST)

hipError_t gemm_ring_launch_i8_small(ecospa_ctx* ctx, const GemmDesc& d, int shape, int k_chunk);

hipError_t gemm_ring_launch_i8(ecospa_ctx* ctx, const GemmDesc& d, int shape) {
  const int k_chunk = (d.K + RING_BK - 1) / RING_BK * RING_BK;
#define I8_CASE(I, BM, BN, NS) if (shape == I) return ring_launch_shape<BM, BN, NS, false, false, false, GEMM_EPIS_I8, false, true>(ctx, d, k_chunk);
  I8_SHAPES(I8_CASE)
  return gemm_ring_launch_i8_small(ctx, d, shape, k_chunk);
}
