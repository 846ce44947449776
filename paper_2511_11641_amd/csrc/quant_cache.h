// Attention over caches of 8-bit floats: descriptors that csrc/quant_cache.hip, csrc/quant_attn.hip and its instantiations share (not part of the C ABI).
#pragma once
#include "common.h"

int ecospa_quant_cache_check(const ecospa_quant_cache* c);

struct QuantAttnArgs {
  const bf16_t* q;
  bf16_t* o;
  float* lse;
  const bf16_t* o_in;
  const float* lse_in;
  const unsigned char *k, *v;
  const float *k_scale, *v_scale;
  const int* lens;
  float* part;                                   // [B][h_kv][row blocks][pieces][rows of a block][kv values, maximum, sum]; NULL: one piece
  long long ld_q, ld_o, ld_oi, k_sb, k_sh, k_st, v_sb, v_sh, v_st;
  int B, L, h, h_kv, g, rows, kq, kv, own_max, block_log2, blocks;      // rows: queries of a request and key/value head, g * L
  int row_blocks, pieces;
  float scale_log2;                              // softmax scale times log2(e)
};
// Most tiles of 16 queries for which accumulators, queries and two groups of keys fit the 256 registers of two wavefronts a SIMD.
static inline constexpr int quant_attn_tiles(int KQ, int W) { return W == 8 || (W == 4 && KQ == 4) ? 2 : 4; }
// Queries of a wavefront in tiles of 16 (T), 32-dim steps of a key (KQ), dims of a value row a lane holds (W: 2, 4 or 8 of 32, 64 or 128); once: one
// item reads a key, and not out of a cache.
hipError_t quant_attn_launch_w2(const QuantAttnArgs& a, int T, int KQ, bool once, hipStream_t st);
hipError_t quant_attn_launch_w4(const QuantAttnArgs& a, int T, int KQ, bool once, hipStream_t st);
hipError_t quant_attn_launch_w8(const QuantAttnArgs& a, int T, int KQ, bool once, hipStream_t st);
