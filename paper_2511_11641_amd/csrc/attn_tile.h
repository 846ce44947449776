// Device code of attention tiles that csrc/attn.hip and csrc/prefix_attn.hip share (not part of the C ABI): fragment types, the swizzled
// LDS layout of [rows][D] key and value tiles, transposing LDS reads and the wait for direct global->LDS loads.
#pragma once
#include "common.h"

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float floatx8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

#define LOG2E 1.4426950408889634f
#define LN2 0.6931471805599453f
#define RESCALE_LOG2 8.0f   // forward softmax: growth of a row maximum (in binades) that triggers a rescale

// ---------------------------------------------------------------------------------------------
// LDS tile addressing (element offsets).  Tiles are [rows][D] (D = 32, 64 or 128 dims, 16-byte chunks
// XOR-swizzled by row) and are read two ways:
//   frag_nat: ds_read_b128, lane (l32, hh) takes chunk 2s+hh of row l32 - sixteen consecutive rows
//             of one chunk column must fall on sixteen different 16-byte bank groups;
//   frag_trn: ds_read_b64_tr_b16, a 16-lane group takes 4 rows x 16 dims - the four rows must fall
//             on four different 64-byte bank groups.
// D = 64 (128-byte rows): swizzle (row % 8) ^ bit 3 of row ^ (bit 1 of row) << 2 serves both;
// D = 32 (64-byte rows, a transposing read covers whole rows): (row / 4) % 4;
// D = 128 (256-byte rows): the swizzle of D = 64 on the low three bits of the chunk number - a bijection of the row's
// sixteen chunks that leaves two-way conflicts on the direct reads (the 128-wide kernels are the rare, wide shapes).
// ---------------------------------------------------------------------------------------------
typedef __attribute__((address_space(3))) bf16_t lds_bf16_t;
typedef short shortx4_t __attribute__((ext_vector_type(4)));
typedef short shortx8_t __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) shortx4_t lds_shortx4_t;

template <int D>
__device__ __forceinline__ int nat_swz(int row) {
  return D >= 64 ? ((row & 7) ^ ((row >> 3) & 1) ^ (((row >> 1) & 1) << 2)) : ((row >> 2) & 3);
}
template <int D>
__device__ __forceinline__ int nat_off(int row, int chunk) {   // [rows][D], D in {32, 64, 128}
  return row * D + ((chunk ^ nat_swz<D>(row)) << 3);
}
template <int D>
__device__ __forceinline__ bf16x8_t frag_nat(const bf16_t* tile, int row, int s, int hh) {
  return *reinterpret_cast<const bf16x8_t*>(tile + nat_off<D>(row, 2 * s + hh));
}
// Operand taken transposed from a natural tile with ds_read_b64_tr_b16: lane (l32, hh) gets dim
// dim0 + l32 of the rows {16s + 4hh + 0..3, 16s + 8 + 4hh + 0..3} - the order in which acc_to_frag()
// lays out the contraction index.  Within a 16-lane group, lane i addresses (row i / 4, dims
// 4 * (i % 4) ..+3) and receives dim i of the group's four rows.
// With two 32-wide sides the reads go out in front of the softmax arithmetic, whose registers leave room for them: their latency passes behind
// it (8 x 1024 causal tokens, 16 heads: dK/dV 47.5 -> 45.3 us, forward 29.6 -> 28.5).
// The reads are issued through inline assembly: the compiler would hold the builtin form back until
// every direct global->LDS load in flight has landed (it cannot tell the stream buffers apart), which
// would undo the prefetch.  The step is an offset in the instruction: these kernels are bound by their vector instructions (62 % of the
// cycles at 32 dims and 1024 tokens, the matrix units 25 %), and addresses were a tenth of them.  trn_issue() starts the two reads of a fragment, trn_wait() waits for all LDS
// reads issued so far, trn_frag() then hands a fragment over (its empty asm statements keep the uses
// behind the wait).
struct TrnRegs { shortx4_t lo, hi; };
template <int D>
__device__ __forceinline__ void trn_issue(TrnRegs& r, const bf16_t* tile, int dim0, int s) {
  const int lane = threadIdx.x & 63, g = lane >> 4, i = lane & 15;
  const int row = 4 * (g >> 1) + (i >> 2);      // the swizzles look at the low four bits of a row: step s is a constant offset
  const int col = dim0 + 16 * (g & 1) + 4 * (i & 3);
  const lds_bf16_t* t3 = (const lds_bf16_t*)tile;
  const unsigned a0 = static_cast<unsigned>(reinterpret_cast<uintptr_t>(t3 + nat_off<D>(row, col >> 3) + (col & 7)));
  const unsigned a1 = static_cast<unsigned>(reinterpret_cast<uintptr_t>(t3 + nat_off<D>(row + 8, col >> 3) + (col & 7)));
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(r.lo) : "v"(a0), "i"(s * 32 * D) : "memory");
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(r.hi) : "v"(a1), "i"(s * 32 * D) : "memory");
}
__device__ __forceinline__ void trn_wait() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ bf16x8_t trn_frag(TrnRegs& r) {
  asm volatile("" : "+v"(r.lo), "+v"(r.hi));
  const shortx8_t v = {r.lo[0], r.lo[1], r.lo[2], r.lo[3], r.hi[0], r.hi[1], r.hi[2], r.hi[3]};
  return __builtin_bit_cast(bf16x8_t, v);
}
// own direct loads have landed (then a barrier tells the same of everyone's)
__device__ __forceinline__ void stream_wait() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0);   // vmcnt(0) lgkmcnt(0) expcnt(0)
  asm volatile("" ::: "memory");
}
