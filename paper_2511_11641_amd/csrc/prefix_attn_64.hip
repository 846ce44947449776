// Attention over a shared prefix and own caches: kernels of heads whose queries and keys have up to 64 dims.
#include "prefix_attn.h"

// explicit instantiation: left to the launch code, the host side of this compiler can drop some of the kernel stubs
#define PREFIX_INSTANTIATE(O, P)                                                     \
  template __global__ void prefix_attn_kernel<64, 32, O, P>(const PrefixArgs);  \
  template __global__ void prefix_attn_kernel<64, 64, O, P>(const PrefixArgs);  \
  template __global__ void prefix_attn_kernel<64, 128, O, P>(const PrefixArgs);
PREFIX_KINDS(PREFIX_INSTANTIATE)
#undef PREFIX_INSTANTIATE

hipError_t prefix_launch_64(const PrefixArgs& a, int dv, int own, int prefix, unsigned grid, hipStream_t st) {
  if (dv == 32) return prefix_launch_width<64, 32>(a, own, prefix, grid, st);
  if (dv == 64) return prefix_launch_width<64, 64>(a, own, prefix, grid, st);
  return prefix_launch_width<64, 128>(a, own, prefix, grid, st);
}
