// Own caches of compact heads: new tokens in (rotated at each request's own position), evicted tokens out (kept rows gathered by the
// accumulated attention weight).  Both move rows of at most 256 bytes and compute next to nothing: bound by memory traffic, or by
// latency alone for the few rows of a decoding step.
#include "common.h"

#include "select_dev.h"
int ecospa_cache_check(const ecospa_cache* c);      // prefix_attn.hip

typedef float kv_floatx8 __attribute__((ext_vector_type(8)));
typedef __bf16 kv_bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned int kv_uintx4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------------------------
// Append: a thread takes 16 bytes of a row of the projection - eight dims of a query, key or value head of one token - turns the four
// pairs in fp32 ((x0, x1) -> (x0 c - x1 s, x0 s + x1 c), rounded once) and writes them to their place.  A thread a piece and no loop: neighbours
// read neighbouring bytes of the row, and write whole rows of a head.  32 x 509 tokens, 32 + 8 + 8 heads of 64 dims turned by tables: 42 us, 200 MB
// of projection and results, 4.8 TB/s beside the tables; one token of four requests 2.2 us, a launch and two latencies.
// ---------------------------------------------------------------------------------------------
struct AppendArgs {
  const bf16_t* qkv;
  bf16_t *q, *k, *v;
  float* weights;
  const float *cos, *sin;
  const int *lens, *pos;
  long long ld_qkv, ld_q, k_sb, k_sh, k_st, v_sb, v_sh, v_st;
  int T, L, L_tab, cap, h, h_kv, g, kq, kv;
  int first_chunk, chunks;      // of a token's row: chunks in front of the first one that is moved (queries that stay where they are), chunks moved
};
__global__ __launch_bounds__(256) void cache_append_kernel(const AppendArgs a) {
  const long long id = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
  const int token = static_cast<int>(id / a.chunks);
  if (token >= a.T) return;
  const int ch = a.first_chunk + static_cast<int>(id - static_cast<long long>(token) * a.chunks);
  const uint4 x = *reinterpret_cast<const uint4*>(a.qkv + token * a.ld_qkv + ch * 8);
  const int b = token / a.L, t = token - b * a.L, slot = a.lens[b] - a.L + t, at = a.cos ? a.pos[b] + t : 0;
  const bool in = slot >= 0 && slot < a.cap && (!a.cos || (at >= 0 && at < a.L_tab));
  const int cq = a.kq >> 3, nq = a.h * cq, nk = a.h_kv * cq, cv = a.kv >> 3;
  if (ch >= nq + nk) {
    const int head = (ch - nq - nk) / cv, d = (ch - nq - nk - head * cv) * 8;
    if (in) *reinterpret_cast<uint4*>(a.v + b * a.v_sb + head * a.v_sh + slot * a.v_st + d) = x;
    return;
  }
  const bool key = ch >= nq;
  const int head = (key ? ch - nq : ch) / cq, d = ((key ? ch - nq : ch) - head * cq) * 8, kh = key ? head : head / a.g;
  uint4 y = x;
  if (a.cos && in) {
    const long long tab = (static_cast<long long>(kh) * a.L_tab + at) * (a.kq >> 1) + (d >> 1);
    const float4 c4 = *reinterpret_cast<const float4*>(a.cos + tab), s4 = *reinterpret_cast<const float4*>(a.sin + tab);
    const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    kv_floatx8 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x0 = __uint_as_float(w[i] << 16), x1 = __uint_as_float(w[i] & 0xffff0000u);
      f[2 * i] = x0 * c[i] - x1 * s[i];
      f[2 * i + 1] = x0 * s[i] + x1 * c[i];
    }
    y = __builtin_bit_cast(uint4, __builtin_convertvector(f, kv_bf16x8));
  }
  if (!key) {
    *reinterpret_cast<uint4*>(a.q + token * a.ld_q + ch * 8) = in ? y : uint4{0u, 0u, 0u, 0u};
  } else if (in) {
    *reinterpret_cast<uint4*>(a.k + b * a.k_sb + head * a.k_sh + slot * a.k_st + d) = y;
    if (a.weights && d == 0) a.weights[(static_cast<long long>(b) * a.h_kv + head) * a.cap + slot] = 0.f;
  }
}

// ---------------------------------------------------------------------------------------------
// Evict.  First launch: a workgroup per (request, key/value head) lists the rows that stay, ascending - the top of the weights of all but the
// last `recent` rows by the radix selection of step 2, then those rows.  Second launch: the gather, 16 bytes a thread.  32 x 8 caches of 8192 rows to
// 2048: 13.4 us (bound by the latency of the selection's passes over 8 MB of weights) and 47.3 us (268 MB, 5.7 TB/s).
// ---------------------------------------------------------------------------------------------
struct EvictArgs {
  const bf16_t *k, *v;
  bf16_t *k_out, *v_out;
  const float* weights;
  float* weights_out;
  const int* lens;
  int *lens_out, *idx;
  long long k_sb, k_sh, k_st, v_sb, v_sh, v_st, ko_sb, ko_sh, ko_st, vo_sb, vo_sh, vo_st;
  int B, h_kv, cap, cap_out, own_max, keep, recent, kq, kv;
  int small;             // pieces are numbered below 2^27: their row is the high half of a product
  unsigned per_inv;      // 2^32 / pieces of a row, rounded up
};
__device__ __forceinline__ int evict_len(const EvictArgs& a, int b) { return min(max(a.lens[b], 0), a.own_max); }
__device__ __forceinline__ void cache_choose(const EvictArgs& a, int bh, SelectShared& sh) {
  const int b = bh / a.h_kv, n = evict_len(a, b);
  int* const idx = a.idx + static_cast<long long>(bh) * a.keep;
  if (threadIdx.x == 0 && bh == b * a.h_kv) a.lens_out[b] = min(n, a.keep);
  if (n <= a.keep) {
    for (int i = threadIdx.x; i < a.keep; i += SELECT_THREADS) idx[i] = i < n ? i : -1;
    return;
  }
  const int old = n - a.recent, top = a.keep - a.recent;
  for (int i = threadIdx.x; i < a.recent; i += SELECT_THREADS) idx[top + i] = old + i;
  if (top == 0) return;
  SelectItemDev t{};
  t.scores = a.weights + static_cast<long long>(bh) * a.cap;
  t.idx = idx;
  t.n = old;
  t.k = top;
  t.groups = 1;
  select_item_block(t, 0, sh);
}
__global__ __launch_bounds__(SELECT_THREADS) void cache_choose_kernel(const EvictArgs a) {
  __shared__ SelectShared sh;
  cache_choose(a, blockIdx.x, sh);
}
// Pieces `id`, id + step, .. of the kept rows of one cache, 16 bytes each, two at a time: row numbers, then rows, then stores, so that two rows of a
// thread are on their way together.  Rows pass once, so neither side is kept in the caches (32 caches of 8192 rows to 2048, 8 heads of 64 + 64 dims,
// 268 MB: one piece at a time 54.8 us, two 53.3, two past the caches 47.5, four 47.6; a plain copy reaches 46).
__device__ __forceinline__ void cache_gather(const EvictArgs& a, int bh, int n, long long id0, long long most, int step) {
  constexpr int U = 2;
  const int b = bh / a.h_kv, hk = bh - b * a.h_kv, cq = a.kq >> 3, per = cq + (a.kv >> 3);
  const int* const idx = a.idx + static_cast<long long>(bh) * a.keep;
  const bf16_t* const k = a.k + b * a.k_sb + hk * a.k_sh;
  const bf16_t* const v = a.v + b * a.v_sb + hk * a.v_sh;
  bf16_t* const ko = a.k_out + b * a.ko_sb + hk * a.ko_sh;
  bf16_t* const vo = a.v_out + b * a.vo_sb + hk * a.vo_sh;
  const float* const w = a.weights + static_cast<long long>(bh) * a.cap;
  float* const wo = a.weights_out ? a.weights_out + static_cast<long long>(bh) * a.cap_out : nullptr;
  const long long all = static_cast<long long>(n) * per, end = all < most ? all : most;
  for (long long id = id0; id < end; id += static_cast<long long>(U) * step) {
    int i[U], c[U], j[U];
    kv_uintx4 x[U];
    float y[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long at = id + static_cast<long long>(u) * step < end ? id + static_cast<long long>(u) * step : id;
      i[u] = static_cast<int>(a.small ? __umulhi(static_cast<unsigned>(at), a.per_inv) : at / per);
      c[u] = static_cast<int>(at - static_cast<long long>(i[u]) * per);
      j[u] = min(max(idx[i[u]], 0), a.cap - 1);      // whatever a list holds, nothing outside the cache is read
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {      // every lane asks for its row's weight: no branch between the loads
      x[u] = __builtin_nontemporal_load(reinterpret_cast<const kv_uintx4*>(c[u] < cq ? k + j[u] * a.k_st + c[u] * 8 : v + j[u] * a.v_st + (c[u] - cq) * 8));
      y[u] = w[j[u]];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (id + static_cast<long long>(u) * step >= end) continue;
      __builtin_nontemporal_store(x[u], reinterpret_cast<kv_uintx4*>(c[u] < cq ? ko + i[u] * a.ko_st + c[u] * 8 : vo + i[u] * a.vo_st + (c[u] - cq) * 8));
      if (c[u] == 0 && wo) wo[i[u]] = y[u];
    }
  }
}
__global__ __launch_bounds__(256) void cache_gather_kernel(const EvictArgs a) {
  const int bh = blockIdx.y, n = min(evict_len(a, bh / a.h_kv), a.keep);
  const long long first = static_cast<long long>(blockIdx.x) * 512;
  cache_gather(a, bh, n, first + threadIdx.x, first + 512, 256);
}
// Both in one launch: the workgroup that chose the rows of a cache moves them.
__global__ __launch_bounds__(SELECT_THREADS) void cache_evict_kernel(const EvictArgs a) {
  __shared__ SelectShared sh;
  cache_choose(a, blockIdx.x, sh);
  __threadfence_block();
  __syncthreads();
  cache_gather(a, blockIdx.x, min(evict_len(a, blockIdx.x / a.h_kv), a.keep), threadIdx.x, 1ll << 62, SELECT_THREADS);
}

// ---------------------------------------------------------------------------------------------
// entry points
// ---------------------------------------------------------------------------------------------
extern "C" int ecospa_cache_append(ecospa_ctx* ctx, const ecospa_cache* c, int L, const void* qkv, long long ld_qkv, const int* pos,
                                   const float* rope_cos, const float* rope_sin, int L_tab, void* q, long long ld_q, float* weights) {
  if (!ctx || !qkv || !rope_cos != !rope_sin || (rope_cos && (!pos || !q))) return ECOSPA_ERR_NULL;
  const int rc = ecospa_cache_check(c);
  if (rc != ECOSPA_OK) return rc;
  const int nq = c->h * c->kp_qk, nk = c->h_kv * c->kp_qk, nv = c->h_kv * c->kp_vo;
  if (L < 1 || static_cast<long long>(c->B) * L * c->h > (1ll << 30) || static_cast<long long>(c->B) * c->h_kv > 65535) return ECOSPA_ERR_SHAPE;
  if (ld_qkv < nq + nk + nv || (q && ld_q < nq) || (rope_cos && L_tab < 1)) return ECOSPA_ERR_SHAPE;
  if (!aligned16(qkv) || ld_qkv % 8 || (q && (!aligned16(q) || ld_q % 8)) || !aligned16(rope_cos) || !aligned16(rope_sin)) return ECOSPA_ERR_ALIGN;
  AppendArgs a;
  memset(&a, 0, sizeof(a));
  a.qkv = static_cast<const bf16_t*>(qkv); a.q = static_cast<bf16_t*>(q); a.k = static_cast<bf16_t*>(c->k); a.v = static_cast<bf16_t*>(c->v);
  a.weights = weights; a.cos = rope_cos; a.sin = rope_sin; a.lens = c->lens; a.pos = pos;
  a.ld_qkv = ld_qkv; a.ld_q = ld_q; a.k_sb = c->k_sb; a.k_sh = c->k_sh; a.k_st = c->k_st; a.v_sb = c->v_sb; a.v_sh = c->v_sh; a.v_st = c->v_st;
  a.T = c->B * L; a.L = L; a.L_tab = L_tab; a.cap = c->cap; a.h = c->h; a.h_kv = c->h_kv; a.g = c->h / c->h_kv; a.kq = c->kp_qk; a.kv = c->kp_vo;
  a.first_chunk = q ? 0 : nq / 8;
  a.chunks = (nq + nk + nv) / 8 - a.first_chunk;
  const long long n = static_cast<long long>(a.T) * a.chunks;
  hipLaunchKernelGGL(cache_append_kernel, dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0, ctx->stream, a);
  ECOSPA_CHECK_LAUNCH(ctx, "cache_append_kernel");
  return ECOSPA_OK;
}

extern "C" int ecospa_cache_evict(ecospa_ctx* ctx, const ecospa_cache* src, const float* weights, int keep, int recent, const ecospa_cache* dst,
                                  int* lens_out, float* weights_out, int* idx) {
  if (!ctx || !src || !dst || !weights || !lens_out || !dst->k || !dst->v) return ECOSPA_ERR_NULL;
  int rc = ecospa_cache_check(src);
  if (rc != ECOSPA_OK) return rc;
  ecospa_cache d = *dst;      // its lengths are an output, its query heads, prefix and bound play no part
  d.lens = lens_out;
  d.h = src->h;
  d.P = 0;
  d.own_max = 0;
  d.scale = src->scale;
  rc = ecospa_cache_check(&d);
  if (rc != ECOSPA_OK) return rc;
  if (d.B != src->B || d.h_kv != src->h_kv || d.kp_qk != src->kp_qk || d.kp_vo != src->kp_vo || static_cast<long long>(src->B) * src->h_kv > 65535)
    return ECOSPA_ERR_SHAPE;
  if (keep < 1 || recent < 0 || recent > keep || d.cap < keep) return ECOSPA_ERR_K;
  if (lens_out == src->lens || weights_out == weights) return ECOSPA_ERR_SHAPE;      // read while they would be written
  EvictArgs a;
  memset(&a, 0, sizeof(a));
  if (!idx) {
    WsCarver ws(ctx->ws, ctx->ws_bytes);
    idx = static_cast<int*>(ws.take(static_cast<size_t>(src->B) * src->h_kv * keep * sizeof(int)));
    if (!ws.ok()) return ECOSPA_ERR_WORKSPACE;
  }
  // rows are gathered by many workgroups at once: what one of them writes, no other may still have to read
  const void* const in[] = {src->k, src->v, src->lens, weights};
  const void* const out[] = {d.k, d.v, lens_out, idx, weights_out};
  for (int i = 0; i < 5; ++i) {
    for (int j = 0; j < 4; ++j)
      if (out[i] == in[j]) return ECOSPA_ERR_SHAPE;
    for (int j = 0; j < i; ++j)
      if (out[i] && out[i] == out[j]) return ECOSPA_ERR_SHAPE;
  }
  a.k = static_cast<const bf16_t*>(src->k); a.v = static_cast<const bf16_t*>(src->v);
  a.k_out = static_cast<bf16_t*>(d.k); a.v_out = static_cast<bf16_t*>(d.v);
  a.weights = weights; a.weights_out = weights_out; a.lens = src->lens; a.lens_out = lens_out; a.idx = idx;
  a.k_sb = src->k_sb; a.k_sh = src->k_sh; a.k_st = src->k_st; a.v_sb = src->v_sb; a.v_sh = src->v_sh; a.v_st = src->v_st;
  a.ko_sb = d.k_sb; a.ko_sh = d.k_sh; a.ko_st = d.k_st; a.vo_sb = d.v_sb; a.vo_sh = d.v_sh; a.vo_st = d.v_st;
  a.B = src->B; a.h_kv = src->h_kv; a.cap = src->cap; a.cap_out = d.cap; a.own_max = src->own_max; a.keep = keep; a.recent = recent;
  a.kq = src->kp_qk; a.kv = src->kp_vo;
  const int groups = a.B * a.h_kv, per = (a.kq + a.kv) / 8;
  const long long n = static_cast<long long>(keep < a.own_max ? keep : a.own_max) * per;      // pieces of a cache
  if ((n + 511) / 512 > 0x7fffffffll) return ECOSPA_ERR_SHAPE;
  a.small = n < 1 << 27;
  a.per_inv = static_cast<unsigned>(((1ll << 32) + per - 1) / per);
  // Small caches: the launch saved outweighs the copying that one workgroup a cache does more slowly (one launch against two, 64 + 64 dims, 4 / 64 /
  // 256 caches: 32 KB each 8.2 / 9.4 / 11.6 us against 8.7 / 9.5 / 12.8, 64 KB 9.4 / 10.5 / 14.3 against 8.8 / 10.7 / 15.3, 128 KB 11.3 / 16.4 / 20.7
  // against 9.0 / 12.3 / 21.9; issued one by one from the host a launch more costs 1.4 us where there is little else).
  if (n * 16 <= 64 * 1024) {
    hipLaunchKernelGGL(cache_evict_kernel, dim3(groups), dim3(SELECT_THREADS), 0, ctx->stream, a);
    ECOSPA_CHECK_LAUNCH(ctx, "cache_evict_kernel");
    return ECOSPA_OK;
  }
  hipLaunchKernelGGL(cache_choose_kernel, dim3(groups), dim3(SELECT_THREADS), 0, ctx->stream, a);
  ECOSPA_CHECK_LAUNCH(ctx, "cache_choose_kernel");
  if (n > 0) {
    hipLaunchKernelGGL(cache_gather_kernel, dim3(static_cast<unsigned>((n + 511) / 512), groups), dim3(256), 0, ctx->stream, a);
    ECOSPA_CHECK_LAUNCH(ctx, "cache_gather_kernel");
  }
  return ECOSPA_OK;
}
