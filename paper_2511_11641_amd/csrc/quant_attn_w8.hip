// Attention over caches of 8-bit floats, value rows of up to 128 dims.
#include "quant_attn.h"

hipError_t quant_attn_launch_w8(const QuantAttnArgs& a, int T, int KQ, bool once, hipStream_t st) { return quant_attn_dispatch<8>(a, T, KQ, once, st); }
