// Attention over a shared prefix and own caches: kernels of heads whose queries and keys have up to 32 dims.
#include "prefix_attn.h"

// explicit instantiation: left to the launch code, the host side of this compiler can drop some of the kernel stubs
#define PREFIX_INSTANTIATE(Q, V, O, P) template __global__ void prefix_attn_kernel<Q, V, O, P>(const PrefixArgs);
PREFIX_KINDS_ALL(PREFIX_INSTANTIATE, 32, 32) PREFIX_KINDS_NARROW(PREFIX_INSTANTIATE, 32, 32)
PREFIX_KINDS_ALL(PREFIX_INSTANTIATE, 32, 64) PREFIX_KINDS_NARROW(PREFIX_INSTANTIATE, 32, 64)
PREFIX_KINDS_ALL(PREFIX_INSTANTIATE, 32, 128) PREFIX_KINDS_WIDE(PREFIX_INSTANTIATE, 32, 128)
#undef PREFIX_INSTANTIATE

hipError_t prefix_launch_32(const PrefixArgs& a, int dv, int own, int prefix, unsigned grid, hipStream_t st) {
  if (dv == 32) return prefix_launch_width<32, 32>(a, own, prefix, grid, st);
  if (dv == 64) return prefix_launch_width<32, 64>(a, own, prefix, grid, st);
  return prefix_launch_width<32, 128>(a, own, prefix, grid, st);
}
