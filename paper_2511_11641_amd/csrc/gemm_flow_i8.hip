// The contraction kernel of resident workgroups for x W^T of 8-bit integers: plain store, GELU (erf), gated.
#include "gemm_flow.h"

#define FLOW_I8(X) X(EPI_STORE) X(EPI_ACT) X(EPI_SWIGLU)
#define FLOW_INST(KIND) template __global__ void gemm_bf16_flow_kernel<FLOW_BM, FLOW_BN, FLOW_NS, false, false, KIND, FLOW_NB, true>(const GemmDesc, int, int);
FLOW_I8(FLOW_INST)

hipError_t gemm_flow_launch_i8(ecospa_ctx* ctx, const GemmDesc& d) {
#define FLOW_CASE(KIND) if (d.epi.kind == KIND) return flow_launch<false, false, KIND, true>(ctx, d);
  FLOW_I8(FLOW_CASE)
  return hipErrorInvalidValue;
}
