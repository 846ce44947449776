// Caches of 8-bit floats (e4m3) with a scale for each block of tokens and head: new tokens in, turned at each request's own position.
#include "quant_cache.h"

typedef float qc_floatx8 __attribute__((ext_vector_type(8)));
typedef __bf16 qc_bf16x8 __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------------------------------------
// Append.  A workgroup takes the new rows that fall into one block of one request's keys or values of a head: its threads hold 8 dims of a row each,
// turned in fp32 and rounded to bf16 (the value a cache of bf16 would keep), agree on the largest and write the codes.  Scales are powers of two,
// the least that keeps the block below the type's 448, so a code is the value's own bits shifted: nothing is lost that the type can hold, and where a block's scale has to rise for a
// new row, the codes of its earlier rows move to it exactly, but for those that fall below the normal range.  Earlier rows that others brought to 8 bits may have another scale, which
// the new ones share unless it has to rise: quotients are divided then.  Further workgroups turn the queries.
// Bound by memory: 32 prompts of 509 tokens, 32 query and 8 key/value heads of 64 dims, 217 MB in 39 us, 5.6 TB/s (a large copy here 5.75); single tokens by the launch.
// ---------------------------------------------------------------------------------------------
struct QuantAppendArgs {
  const bf16_t* qkv;
  bf16_t* q;
  unsigned char *k, *v;
  float *k_scale, *v_scale;
  const float *cos, *sin;
  const int *lens, *pos;
  long long ld_qkv, ld_q, k_sb, k_sh, k_st, v_sb, v_sh, v_st, n_queries;
  int B, L, L_tab, cap, h, h_kv, g, kq, kv, block, blocks, touched;      // blocks: of a cache; touched: that the rows of a call can fall into
  int n_items;                                                           // workgroups that put rows into the cache
};
// 8 dims of a head turned by its angles of one position, rounded to bf16.  Which product is fused is written out: the bits are those that the append
// into caches of bf16 gives.
__device__ __forceinline__ uint4 quant_turn(const uint4& x, const float* cos, const float* sin) {
  const float4 c4 = *reinterpret_cast<const float4*>(cos), s4 = *reinterpret_cast<const float4*>(sin);
  const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  qc_floatx8 f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x0 = __uint_as_float(w[i] << 16), x1 = __uint_as_float(w[i] & 0xffff0000u);
    f[2 * i] = __builtin_fmaf(x0, c[i], -__fmul_rn(x1, s[i]));
    f[2 * i + 1] = __builtin_fmaf(x0, s[i], __fmul_rn(x1, c[i]));
  }
  return __builtin_bit_cast(uint4, __builtin_convertvector(f, qc_bf16x8));
}
// The least power of two (2^-100 and above) with |x| <= 448 times it, for the finite x >= 0 of these bits: 448 is 1.75 * 2^8.
__device__ __forceinline__ float quant_scale_for(unsigned bits) {
  const int e = static_cast<int>(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return __uint_as_float(static_cast<unsigned>(max(e, -100) + 127) << 23);
}
// four values, brought to a block's scale by `to`, to codes; what is not finite becomes NaN (the type has no infinity)
template <typename F>
__device__ __forceinline__ unsigned quant_pack4(float a, float b, float c, float d, F&& to) {
  const auto put = [&](float x) __attribute__((always_inline)) { return fabsf(x) < INFINITY ? to(x) : __uint_as_float(0x7fc00000u); };
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(put(a), put(b), 0, false);
  return static_cast<unsigned>(__builtin_amdgcn_cvt_pk_fp8_f32(put(c), put(d), w, true));
}
// y, the nearest number to y + rest, as the neighbour of y + rest whose last bit is set: its rounding to a code's four bits is then that of y + rest, not that of a half way
// which y only rounds to
__device__ __forceinline__ float quant_sticky(float y, float rest) {
  const unsigned u = __float_as_uint(y);
  return y == 0.f || rest == 0.f ? y : __uint_as_float(((u ^ __float_as_uint(rest)) >> 31 ? u - 1u : u) | 1u);
}
template <int THREADS, int EACH>
__global__ __launch_bounds__(THREADS) void quant_append_kernel(const QuantAppendArgs a) {
  const int t = threadIdx.x;
  if (static_cast<int>(blockIdx.x) >= a.n_items) {      // queries, 8 dims a thread
    const long long id = static_cast<long long>(blockIdx.x - a.n_items) * THREADS + t;
    if (id >= a.n_queries) return;
    const int cq = a.kq >> 3, per = a.h * cq, token = static_cast<int>(id / per), ch = static_cast<int>(id - static_cast<long long>(token) * per);
    const int b = token / a.L, slot = a.lens[b] - a.L + token - b * a.L, at = a.cos ? a.pos[b] + token - b * a.L : 0, head = ch / cq;
    const bool in = slot >= 0 && slot < a.cap && (!a.cos || (at >= 0 && at < a.L_tab));
    uint4 x = *reinterpret_cast<const uint4*>(a.qkv + token * a.ld_qkv + ch * 8);
    if (a.cos && in) {
      const long long tab = (static_cast<long long>(head / a.g) * a.L_tab + at) * (a.kq >> 1) + (ch - head * cq) * 4;
      x = quant_turn(x, a.cos + tab, a.sin + tab);
    }
    *reinterpret_cast<uint4*>(a.q + token * a.ld_q + ch * 8) = in ? x : uint4{0u, 0u, 0u, 0u};
    return;
  }
  int id = blockIdx.x;
  const bool key = id & 1;
  id >>= 1;
  const int i = id % a.touched;
  id /= a.touched;
  const int b = id / a.h_kv, head = id - b * a.h_kv;
  const int at0 = a.cos ? a.pos[b] : 0;                                  // position of the first new token
  const int first = a.lens[b] - a.L, end = min(first + a.L, a.cap);      // rows of the new tokens
  const int blk = max(first, 0) / a.block + i, row0 = blk * a.block;
  const int lo = max(max(first, 0), row0), hi = min(end, row0 + a.block);
  if (lo >= hi) return;
  const int width = key ? a.kq : a.kv, cw = width >> 3, pieces = (hi - lo) * cw;
  const bf16_t* const src = a.qkv + a.h * a.kq + (key ? head * a.kq : a.h_kv * a.kq + head * a.kv);
  float* const at_scale = (key ? a.k_scale : a.v_scale) + (static_cast<long long>(b) * a.h_kv + head) * a.blocks + blk;
  const bool earlier = lo > row0;
  const float before = earlier ? *at_scale : 0.f;
  uint4 x[EACH];
  bool in[EACH];
  unsigned top = 0u;
#pragma unroll
  for (int c = 0; c < EACH; ++c) {
    const int p = min(c * THREADS + t, pieces - 1), r = p / cw, d = p - r * cw, at = at0 + lo - first + r;
    in[c] = c * THREADS + t < pieces;
    x[c] = *reinterpret_cast<const uint4*>(src + (static_cast<long long>(b) * a.L + lo - first + r) * a.ld_qkv + d * 8);
    if (a.cos) in[c] = in[c] && at >= 0 && at < a.L_tab;
    if (key && a.cos && in[c]) {
      const long long tab = (static_cast<long long>(head) * a.L_tab + at) * (a.kq >> 1) + d * 4;
      x[c] = quant_turn(x[c], a.cos + tab, a.sin + tab);
    }
    top = in[c] ? max(top, 1u) : top;
    const unsigned w[4] = {x[c].x, x[c].y, x[c].z, x[c].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const unsigned u = (w[e] << 16) & 0x7fffffffu, v = w[e] & 0x7fff0000u;
      top = in[c] && u < 0x7f800000u ? max(top, u) : top;
      top = in[c] && v < 0x7f800000u ? max(top, v) : top;
    }
  }
  top = ~wave_umin(~top);
  if constexpr (THREADS > 64) {
    __shared__ unsigned red[THREADS / 64];
    if ((t & 63) == 0) red[t >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) top = max(top, red[w]);
  }
  if (top == 0u) return;      // no row of the block has an angle: nothing changes
  const float s = fmaxf(quant_scale_for(top), before);
  unsigned char* const dst = (key ? a.k + b * a.k_sb + head * a.k_sh : a.v + b * a.v_sb + head * a.v_sh);
  const long long st = key ? a.k_st : a.v_st;
  if (earlier && s > before) {      // the earlier rows come to the new scale
    const float r = before / s;      // exact: s is a power of two
    for (int p = t; p < (lo - row0) * cw; p += THREADS) {
      const int row = p / cw, d = p - row * cw;
      uint2* const at = reinterpret_cast<uint2*>(dst + (row0 + row) * st + d * 8);
      const uint2 u = *at;
      unsigned w[2] = {u.x, u.y};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const auto f = __builtin_amdgcn_cvt_pk_f32_fp8(w[e], false), g = __builtin_amdgcn_cvt_pk_f32_fp8(w[e], true);
        w[e] = quant_pack4(f[0], f[1], g[0], g[1], [r](float c) __attribute__((always_inline)) { const float y = c * r; return quant_sticky(y, __builtin_fmaf(c, r, -y)); });
      }
      *at = make_uint2(w[0], w[1]);
    }
  }
  if (THREADS > 64) __syncthreads();      // everyone has read the scale of before
  if (t == 0) *at_scale = s;
  const auto store = [&](auto&& to) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < EACH; ++c) {
      if (!in[c]) continue;
      const int p = c * THREADS + t, row = p / cw, d = p - row * cw;
      const unsigned w[4] = {x[c].x, x[c].y, x[c].z, x[c].w};
      float f[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) { f[2 * e] = __uint_as_float(w[e] << 16); f[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
      *reinterpret_cast<uint2*>(dst + (lo + row) * st + d * 8) = make_uint2(quant_pack4(f[0], f[1], f[2], f[3], to), quant_pack4(f[4], f[5], f[6], f[7], to));
    }
  };
  if ((__float_as_uint(s) & 0x7fffffu) == 0u) {      // a power of two, exactly
    const float r = 1.f / s;
    store([r](float v) __attribute__((always_inline)) { return v * r; });
  } else {      // (both scaled by 2^64 where s is small, so that no remainder is lost below the least number)
    const float up = s < 1.f ? 0x1p64f : 1.f, d = s * up;
    store([up, d](float v) __attribute__((always_inline)) { const float n = v * up, y = n / d; return quant_sticky(y, __builtin_fmaf(-y, d, n)); });
  }
}

// ---------------------------------------------------------------------------------------------
// entry points
// ---------------------------------------------------------------------------------------------
int ecospa_quant_cache_check(const ecospa_quant_cache* c) {
  if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale || !c->lens) return ECOSPA_ERR_NULL;
  if (c->B < 1 || c->h < 1 || c->h_kv < 1 || c->h % c->h_kv || c->cap < 1 || c->own_max < 0 || c->own_max > c->cap) return ECOSPA_ERR_SHAPE;
  if (c->kp_qk < 16 || c->kp_qk > 128 || c->kp_qk % 16 || c->kp_vo < 16 || c->kp_vo > 128 || c->kp_vo % 16) return ECOSPA_ERR_SHAPE;
  if (c->block < 16 || c->block > 128 || (c->block & (c->block - 1)) || !(c->scale > 0.f && c->scale < INFINITY)) return ECOSPA_ERR_SHAPE;
  if (c->k_st < c->kp_qk || c->v_st < c->kp_vo || c->k_st >= 1 << 25 || c->v_st >= 1 << 25 || c->k_sb < 0 || c->k_sh < 0 || c->v_sb < 0 || c->v_sh < 0) return ECOSPA_ERR_SHAPE;
  if (static_cast<long long>(c->B) * c->h_kv > 65535) return ECOSPA_ERR_SHAPE;
  if (!aligned16(c->k) || !aligned16(c->v) || c->k_sb % 16 || c->k_sh % 16 || c->k_st % 16 || c->v_sb % 16 || c->v_sh % 16 || c->v_st % 16 ||
      (reinterpret_cast<uintptr_t>(c->k_scale) & 3u) || (reinterpret_cast<uintptr_t>(c->v_scale) & 3u) || (reinterpret_cast<uintptr_t>(c->lens) & 3u))
    return ECOSPA_ERR_ALIGN;
  return ECOSPA_OK;
}

extern "C" int ecospa_quant_cache_append(ecospa_ctx* ctx, const ecospa_quant_cache* c, int L, const void* qkv, long long ld_qkv, const int* pos,
                                         const float* rope_cos, const float* rope_sin, int L_tab, void* q, long long ld_q) {
  if (!ctx || !qkv || !rope_cos != !rope_sin || (rope_cos && (!pos || !q))) return ECOSPA_ERR_NULL;
  const int rc = ecospa_quant_cache_check(c);
  if (rc != ECOSPA_OK) return rc;
  const int nq = c->h * c->kp_qk, nk = c->h_kv * c->kp_qk, nv = c->h_kv * c->kp_vo;
  if (L < 1 || static_cast<long long>(c->B) * L * c->h > (1ll << 30)) return ECOSPA_ERR_SHAPE;
  if (ld_qkv < nq + nk + nv || (q && ld_q < nq) || (rope_cos && L_tab < 1)) return ECOSPA_ERR_SHAPE;
  if (!aligned16(qkv) || ld_qkv % 8 || (q && (!aligned16(q) || ld_q % 8)) || !aligned16(rope_cos) || !aligned16(rope_sin)) return ECOSPA_ERR_ALIGN;
  QuantAppendArgs a;
  memset(&a, 0, sizeof(a));
  a.qkv = static_cast<const bf16_t*>(qkv); a.q = static_cast<bf16_t*>(q); a.k = static_cast<unsigned char*>(c->k); a.v = static_cast<unsigned char*>(c->v);
  a.k_scale = c->k_scale; a.v_scale = c->v_scale; a.cos = rope_cos; a.sin = rope_sin; a.lens = c->lens; a.pos = pos;
  a.ld_qkv = ld_qkv; a.ld_q = ld_q; a.k_sb = c->k_sb; a.k_sh = c->k_sh; a.k_st = c->k_st; a.v_sb = c->v_sb; a.v_sh = c->v_sh; a.v_st = c->v_st;
  a.B = c->B; a.L = L; a.L_tab = L_tab; a.cap = c->cap; a.h = c->h; a.h_kv = c->h_kv; a.g = c->h / c->h_kv; a.kq = c->kp_qk; a.kv = c->kp_vo;
  a.block = c->block;
  a.blocks = (c->cap + c->block - 1) / c->block;
  a.touched = (L + 2 * (c->block - 1)) / c->block;
  if (a.touched > a.blocks) a.touched = a.blocks;
  const long long items = 2ll * c->B * c->h_kv * a.touched;
  a.n_queries = q ? static_cast<long long>(c->B) * L * (nq / 8) : 0;
  if (items > (1ll << 30)) return ECOSPA_ERR_SHAPE;
  a.n_items = static_cast<int>(items);
  const int pieces = (L < c->block ? L : c->block) * (c->kp_qk > c->kp_vo ? c->kp_qk : c->kp_vo) / 8;
  // a wavefront a block up to 256 pieces, one each up to 64 (us, 32 prompts of 16 tokens 5.9 : 6.1; against a workgroup of 256: of 400 tokens, 16 heads of 32 dims
  // and blocks of 32, 15 : 30; single tokens 5.9 : 6.3), else a workgroup, with registers for no more than
  // the block has (32 prompts of 509 tokens and 64 dims: blocks of 64, room for 2, 4 and 8 pieces a thread 39 : 43 : 56; of 128, 4 and 8 37.5 : 47)
  const int threads = pieces <= 256 ? 64 : 256;
  const long long grid = items + (a.n_queries + threads - 1) / threads;
  if (grid * threads >= 1ll << 32) return ECOSPA_ERR_SHAPE;      // a launch takes no more work-items
  const dim3 g(static_cast<unsigned>(grid)), n(threads);
  if (pieces <= 64) hipLaunchKernelGGL((quant_append_kernel<64, 1>), g, n, 0, ctx->stream, a);
  else if (pieces <= 256) hipLaunchKernelGGL((quant_append_kernel<64, 4>), g, n, 0, ctx->stream, a);
  else if (pieces <= 512) hipLaunchKernelGGL((quant_append_kernel<256, 2>), g, n, 0, ctx->stream, a);
  else if (pieces <= 1024) hipLaunchKernelGGL((quant_append_kernel<256, 4>), g, n, 0, ctx->stream, a);
  else hipLaunchKernelGGL((quant_append_kernel<256, 8>), g, n, 0, ctx->stream, a);
  ECOSPA_CHECK_LAUNCH(ctx, "quant_append_kernel");
  return ECOSPA_OK;
}
